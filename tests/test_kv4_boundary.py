"""Calls on a 4-bit key/value cache: arguments that are refused on the host, before anything is launched.  No GPU needed."""
import ctypes

import pytest
import torch

import paper_2512_05746_amd as hq
from paper_2512_05746_amd.binding import _Kv4

OK, NULL, SHAPE, DTYPE, BITS, ALIGN, UNSUPPORTED = range(7)
P = 4096   # any non-null, 16-byte-aligned fake device address: validation never dereferences it
F16, F32, I32, BF16 = range(4)
STRIDES = (ctypes.c_int64 * 8)(*[512] * 8)


@pytest.fixture(scope="module")
def lib():
    return hq.load_library()


def cache(**kw):
    c = dict(k=P, v=P, k_scale=P, v_scale=P, page_table=P, lengths=P, begins=P, pages=10, t=0, page_size=16, kv_heads=2, d=64, had_block=64, batch=2,
             table_pages=4)
    c.update(kw)
    return ctypes.byref(_Kv4(**c))


def calls(lib):
    def append(c=None, q=P, k=P, v=P, dt=F16, heads=4, strides=STRIDES, qw=None, kw=None, wdt=F16, cos=P, sin=P, positions=8, rotary=64, interleaved=0, pos=None,
               pos_size=0, norm=1, eps=1e-6, out=P, **cache_kw):
        return lib.hq_kv4_append(c or cache(**cache_kw), q, k, v, dt, heads, strides, qw, kw, wdt, cos, sin, positions, rotary, interleaved, pos, pos_size, norm, eps,
                                 out, None)

    def attention(q=P, dt=F16, heads=4, strides=STRIDES, scale=0.1, window=0, sinks=0, space=P, out=P, **cache_kw):
        return lib.hq_kv4_attention(cache(**cache_kw), q, dt, heads, strides, scale, window, sinks, space, out, None)

    def read(k=P, v=P, dt=F16, **cache_kw):
        return lib.hq_kv4_read(cache(**cache_kw), k, v, dt, None)

    return append, attention, read


def test_cache_arguments(lib):
    for call in calls(lib):
        assert call() == OK                                             # no tokens: nothing launched
        assert call(k_scale=None, page_table=None, lengths=None, begins=None) == OK
        for name in ("v_scale", "k_scale", "page_table", "lengths"):
            assert call(t=4, **{name: None}) == NULL, name
        for bad in (dict(kv_heads=0), dict(kv_heads=-1), dict(d=0), dict(d=60), dict(pages=0), dict(batch=-1),
                    dict(table_pages=0), dict(t=-1), dict(page_size=0), dict(page_size=24), dict(had_block=0), dict(had_block=3), dict(had_block=128),
                    dict(batch=0, t=4), dict(begins=None, t=3)):
            assert call(**bad) == SHAPE, bad
        for bad in (dict(d=264, had_block=8), dict(page_size=4), dict(d=256, had_block=256), dict(table_pages=1 << 27), dict(t=1 << 30, begins=P),
                    dict(pages=1 << 60)):
            assert call(**bad) == UNSUPPORTED, bad
        for bad in (dict(v_scale=P + 8), dict(k_scale=P + 4), dict(page_table=P + 2), dict(lengths=P + 1), dict(begins=P + 2)):
            assert call(**bad) == ALIGN, bad
        assert call(dt=I32) == DTYPE and call(dt=9) == DTYPE


def test_more_than_a_launch_holds(lib):
    many = dict(t=8 * 0x500000 + 8, kv_heads=1)
    for call in calls(lib):
        assert call(**many) == UNSUPPORTED and call(t=8, batch=0x300000) == UNSUPPORTED
    _, attention, _ = calls(lib)
    assert attention(heads=32, t=40_000_000, d=256, had_block=128) == UNSUPPORTED   # 16 x 40e6 rows of 2 heads, 64 to 256 lanes


def test_append_arguments(lib):
    append, _, _ = calls(lib)
    assert lib.hq_kv4_append(None, P, P, P, F16, 4, STRIDES, None, None, F16, P, P, 8, 64, 0, None, 0, 1, 1e-6, P, None) == NULL
    assert append(strides=None) == NULL and append(cos=None) == NULL and append(sin=None) == NULL
    for name in ("q", "k", "v", "out"):
        assert append(**{name: None}, c=cache(t=4)) == NULL
    assert append(heads=3) == SHAPE and append(heads=0) == SHAPE
    assert append(rotary=66) == SHAPE and append(rotary=3) == SHAPE and append(rotary=-2) == SHAPE and append(positions=0) == SHAPE
    assert append(eps=-1.0) == SHAPE and append(eps=float("nan")) == SHAPE and append(eps=-1.0, norm=0) == OK
    assert append(norm=0, qw=P) == SHAPE and append(norm=0, kw=P) == SHAPE
    assert append(wdt=BF16) == DTYPE and append(wdt=F32) == OK and append(pos=P, pos_size=2) == DTYPE
    assert append(q=P + 1) == ALIGN and append(dt=F32, wdt=F32, c=cache(), out=P + 2) == ALIGN and append(cos=P + 2) == ALIGN and append(pos=P + 4, pos_size=8) == ALIGN
    assert append(qw=P + 1) == ALIGN and append(kw=P + 2, wdt=F32) == ALIGN
    assert append(rotary=0, cos=None, sin=None) == OK


def test_attention_arguments(lib):
    _, attention, _ = calls(lib)
    assert lib.hq_kv4_attention(None, P, F16, 4, STRIDES, 0.1, 0, 0, P, P, None) == NULL
    assert attention(strides=None) == NULL and attention(t=4, q=None) == NULL and attention(t=4, out=None) == NULL
    assert attention(heads=5) == SHAPE and attention(window=-1) == SHAPE and attention(sinks=-1) == SHAPE
    assert attention(scale=float("nan")) == SHAPE and attention(scale=float("inf")) == SHAPE and attention(scale=1e31) == SHAPE
    assert attention(q=P + 1) == ALIGN and attention(out=P + 1) == ALIGN
    long = dict(t=2, table_pages=4096, begins=None)
    size = lambda **kw: lib.hq_kv4_attention_workspace(cache(**{**long, **kw}), F16, 4, 0, 0)
    assert size() > 0 and attention(space=None, **long) == NULL and attention(space=P + 4, **long) == ALIGN
    assert size(t=0) >= 0 and size(d=60) == 0 and size(table_pages=1) == 0     # one short page: nothing to join
    assert lib.hq_kv4_attention_workspace(None, F16, 4, 0, 0) == 0 and lib.hq_kv4_attention_workspace(cache(), I32, 4, 0, 0) == 0


def test_read_arguments(lib):
    _, _, read = calls(lib)
    assert lib.hq_kv4_read(None, P, P, F16, None) == NULL
    assert read(dt=F32, k=P, v=P, t=0) == OK


def test_python_refuses():
    c = hq.hq_kv4_cache(4, 16, 2, 64, device="cpu")
    assert c.k.shape == (4, 2, 16, 32) and c.v.shape == (4, 2, 2, 64, 4) and c.k_scale.shape == c.v_scale.shape == (4, 2, 16)
    assert hq.hq_kv4_cache(1, 8, 1, 72, device="cpu").v.shape == (1, 1, 1, 96, 4)
    table, lengths = torch.zeros(1, 4, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q, none = torch.zeros(1, 4, 64), torch.zeros(1, 0)
    with pytest.raises(ValueError):
        hq.hq_kv4_attention(q, c, table, lengths)
    with pytest.raises(ValueError):
        hq.hq_kv4_read(c, table, lengths, 1)
    with pytest.raises(ValueError):
        hq.hq_kv4_append(q, q[:, :2], q[:, :2], None, None, none, none, c, table, lengths)
    with pytest.raises(TypeError):
        hq.hq_kv4_attention(None, c, table, lengths)
