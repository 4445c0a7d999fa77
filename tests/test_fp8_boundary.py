"""Calls on 8-bit floats and on query and key heads: arguments that are refused on the host, before anything is launched.  No GPU needed."""
import ctypes

import pytest
import torch

import paper_2512_05746_amd as hq

OK, NULL, SHAPE, DTYPE, BITS, ALIGN, UNSUPPORTED = range(7)
P = 4096   # any non-null, 16-byte-aligned fake device address: validation never dereferences it
F16, F32, I32, BF16 = range(4)


@pytest.fixture(scope="module")
def lib():
    return hq.load_library()


def call_of(f, names):
    """f with defaults by name."""
    return lambda **kw: f(*[kw.get(n, d) for n, d in names])


def test_quantiser_arguments(lib):
    rows = call_of(lib.hq_fp8_quantize_rows, [("x", P), ("dt", F16), ("m", 8), ("k", 200), ("stride", 200), ("xq", P), ("s", P), ("st", None)])
    assert rows(x=None) == NULL and rows(xq=None) == NULL and rows(s=None) == NULL
    assert rows(dt=I32) == DTYPE and rows(dt=9) == DTYPE
    assert rows(m=-1) == SHAPE and rows(k=0) == SHAPE and rows(stride=-1) == SHAPE
    assert rows(x=P + 1) == ALIGN and rows(dt=F32, x=P + 2) == ALIGN and rows(xq=P + 8) == ALIGN and rows(s=P + 2) == ALIGN
    assert rows(m=65536 * 128) == UNSUPPORTED
    assert rows(m=0) == OK and rows(m=0, x=None, xq=None, s=None) == OK   # nothing to do, nothing launched
    blocks = call_of(lib.hq_fp8_quantize_blocks, [("w", P), ("dt", BF16), ("n", 8), ("k", 200), ("stride", 200), ("wq", P), ("wt", P), ("s", P), ("st", None)])
    assert blocks(w=None) == NULL and blocks(wq=None, wt=None) == NULL and blocks(s=None) == NULL
    assert blocks(dt=I32) == DTYPE
    assert blocks(n=0) == SHAPE and blocks(k=0) == SHAPE
    assert blocks(w=P + 1) == ALIGN and blocks(wq=P + 4) == ALIGN and blocks(wt=P + 4) == ALIGN


def test_linear_arguments(lib):
    linear = call_of(lib.hq_fp8_linear, [("xq", P), ("sx", P), ("wq", P), ("sw", P), ("turned", 0), ("bias", None), ("m", 8), ("n", 24), ("k", 200), ("y", P),
                                         ("dt", BF16), ("st", None)])
    for name in ("xq", "sx", "wq", "sw", "y"):
        assert linear(**{name: None}) == NULL
    assert linear(dt=I32) == DTYPE
    assert linear(m=-1) == SHAPE and linear(n=0) == SHAPE and linear(k=0) == SHAPE
    assert linear(xq=P + 8) == ALIGN and linear(wq=P + 8) == ALIGN and linear(y=P + 1) == ALIGN and linear(dt=F32, y=P + 2) == ALIGN and linear(bias=P + 1) == ALIGN
    assert linear(k=1 << 23) == UNSUPPORTED and linear(m=1 << 40, n=1 << 20) == UNSUPPORTED
    assert linear(m=0, xq=None, sx=None, y=None) == OK
    layer = call_of(lib.hq_act_quant_fp8_linear, [("x", P), ("xdt", F16), ("stride", 4096), ("wq", P), ("sw", P), ("bias", None), ("m", 4096), ("n", 4096),
                                                  ("k", 4096), ("space", P), ("y", P), ("dt", F16), ("st", None)])
    assert layer(x=None) == NULL and layer(wq=None) == NULL and layer(sw=None) == NULL and layer(y=None) == NULL
    assert layer(xdt=I32) == DTYPE and layer(dt=I32) == DTYPE
    assert layer(stride=-4) == SHAPE and layer(n=0) == SHAPE
    assert layer(space=P + 8) == ALIGN
    size = lib.hq_act_quant_fp8_linear_workspace(F16, 4096, 4096, 4096, F16)
    assert size == 4096 * 4096 + 4 * 32 * 4096
    assert layer(space=None) == NULL                                        # a layer of two launches needs it
    assert lib.hq_act_quant_fp8_linear_workspace(F16, 1, 960, 960, F16) == 0   # one launch: no workspace
    assert lib.hq_act_quant_fp8_linear_workspace(F16, 0, 960, 960, F16) == 0


def test_backward_arguments(lib):
    back = call_of(lib.hq_fp8_linear_backward, [("dy", P), ("dys", 24), ("x", P), ("xs", 200), ("dt", F16), ("wt", P), ("sw", P), ("m", 8), ("n", 24), ("k", 200),
                                                ("space", P), ("dx", P), ("dw", P), ("db", None), ("st", None)])
    for name in ("dy", "x", "wt", "sw", "space", "dx", "dw"):
        assert back(**{name: None}) == NULL
    assert back(dt=I32) == DTYPE
    assert back(m=-1) == SHAPE and back(n=0) == SHAPE and back(dys=-1) == SHAPE and back(xs=-1) == SHAPE
    assert back(wt=P + 8) == ALIGN and back(space=P + 8) == ALIGN and back(dw=P + 2) == ALIGN and back(db=P + 2) == ALIGN and back(dx=P + 1) == ALIGN
    assert back(n=1 << 23) == UNSUPPORTED and back(m=1 << 24) == UNSUPPORTED
    assert lib.hq_fp8_linear_backward_workspace(0, 24, 200) == 0
    assert lib.hq_fp8_linear_backward_workspace(300, 264, 520) >= 300 * 272 + 264 * 304 + 520 * 304


def test_heads_arguments(lib):
    strides = (ctypes.c_int64 * 12)(*([512, 64] * 6))
    names = [("dt", F16), ("t", 8), ("h", 4), ("hk", 2), ("d", 64), ("strides", strides), ("qw", P), ("kw", P), ("wdt", F16), ("cos", P), ("sin", P), ("pos_n", 16),
             ("r", 64), ("inter", 0), ("pos", P), ("ps", 8), ("eps", 1e-6)]
    heads = call_of(lib.hq_qk_norm_rope, [("q", P), ("k", P)] + names + [("qo", P), ("ko", P), ("st", None)])
    back = call_of(lib.hq_qk_norm_rope_backward, [("dq", P), ("dk", P), ("q", P), ("k", P)] + names + [("space", P), ("qo", P), ("ko", P), ("dqw", P), ("dkw", P),
                                                                                                      ("st", None)])
    for f, pointers in ((heads, ("q", "k", "qo", "ko")), (back, ("dq", "dk", "q", "k", "qo", "ko", "space"))):
        for name in pointers + ("strides", "cos", "sin"):
            assert f(**{name: None}) == NULL
        assert f(dt=I32) == DTYPE and f(wdt=BF16) == DTYPE and f(ps=2) == DTYPE
        assert f(t=-1) == SHAPE and f(h=0) == SHAPE and f(hk=0) == SHAPE and f(d=63, r=62) == SHAPE and f(r=33) == SHAPE and f(r=66) == SHAPE
        assert f(pos=None, t=17) == SHAPE                 # no positions, and tables that are too short
        assert f(eps=-1.0) == SHAPE and f(eps=float("nan")) == SHAPE and f(pos_n=0) == SHAPE
        assert f(d=1026, r=64) == UNSUPPORTED and f(t=1 << 30) == UNSUPPORTED
        assert f(q=P + 1) == ALIGN and f(ko=P + 1) == ALIGN and f(qw=P + 1) == ALIGN and f(cos=P + 2) == ALIGN and f(pos=P + 4) == ALIGN
    assert heads(t=0, q=None, k=None, qo=None, ko=None) == OK
    assert back(space=P + 2) == ALIGN and back(dqw=P + 2) == ALIGN
    assert lib.hq_qk_norm_rope_backward_workspace(F16, 8, 4, 2, 63, 62) == 0
    assert lib.hq_qk_norm_rope_backward_workspace(F16, 8, 4, 2, 64, 64) >= 2 * 64 * 4


def test_calls_on_integer_codes_do_not_take_bfloat16(lib):
    assert lib.hq_act_hadamard_quant(P, BF16, 8, 64, 64, 4, P, P, None) == DTYPE
    assert lib.hq_quantize_weights(P, BF16, 8, 1, 64, 64, 4, P, P, None) == DTYPE
    assert lib.hq_int_linear(P, P, P, P, None, 8, 8, 64, P, BF16, None) == DTYPE
    assert lib.hq_int_linear_i8(P, P, P, P, None, 8, 8, 64, P, BF16, None) == DTYPE
    assert lib.hq_int_conv2d(P, P, P, P, None, 1, 4, 4, 64, 8, 3, 3, 1, 1, P, BF16, None) == DTYPE
    assert lib.hq_act_quant_int_linear(P, BF16, P, P, None, 8, 8, 64, 64, 4, P, F16, None, None, None) == DTYPE


def test_binding_rejects_host_tensors():
    x, q = torch.zeros(4, 32), torch.zeros(4, 2, 32)
    codes = torch.zeros(4, 32, dtype=torch.uint8).view(torch.float8_e4m3fn)
    one = torch.ones(1, 4)
    for call in (lambda: hq.hq_fp8_quantize_rows(x), lambda: hq.hq_fp8_quantize_blocks(x), lambda: hq.hq_fp8_linear(codes, one, codes, one),
                 lambda: hq.hq_act_quant_fp8_linear(x, codes, one), lambda: hq.hq_fp8_linear_backward(x, x, codes, one),
                 lambda: hq.hq_qk_norm_rope(q, q, None, None, one, one), lambda: hq.hq_qk_norm_rope_backward(q, q, q, q, None, None, one, one)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: hq.hq_fp8_quantize_rows(None), lambda: hq.hq_qk_norm_rope(None, q, None, None, one, one)):
        with pytest.raises(TypeError):
            call()


def test_gradients_of_heads_that_do_not_fit_name_the_reason(lib):
    """Their workspace has no bytes, so it may be no memory at all: the sizes are what is wrong."""
    strides = (ctypes.c_int64 * 12)(*([4096, 64] * 6))

    def back(d=64, rotary=64, t=8, heads=4, space=None, positions=16):
        return lib.hq_qk_norm_rope_backward(P, P, P, P, F16, t, heads, 2, d, strides, P, P, F16, P, P, positions, rotary, 0, P, 8, 1e-6, space, P, P, P, P,
                                            None)

    assert back(d=63, rotary=62) == SHAPE and back(rotary=66) == SHAPE and back(rotary=33) == SHAPE and back(positions=0) == SHAPE
    assert back(d=1026) == UNSUPPORTED and back(t=1 << 29) == UNSUPPORTED
    for d, rotary, t in ((63, 62, 8), (64, 66, 8), (1026, 64, 8), (64, 64, 1 << 29)):
        assert lib.hq_qk_norm_rope_backward_workspace(F16, t, 4, 2, d, rotary) == 0
    assert back() == NULL   # sizes that fit need it


def test_calls_that_record_no_gradient_refuse_tensors_that_need_one():
    """While gradients are recorded; under no_grad, and for weights that are quantised, the tensors are taken.  (Fake device tensors: the call
    ends with an error of another kind, since they have no memory.)"""
    from torch._subclasses.fake_tensor import FakeTensor, FakeTensorMode
    mode = FakeTensorMode()

    def fake(*shape, dtype=torch.float16, grad=False):
        t = FakeTensor(mode, torch.empty(shape, dtype=dtype, device="meta"), torch.device("cuda"))
        return t.requires_grad_() if grad else t

    codes = lambda *shape: fake(*shape, dtype=torch.float8_e4m3fn)
    f32 = lambda *shape: fake(*shape, dtype=torch.float32)
    layer = lambda x, b: hq.hq_act_quant_fp8_linear(x, codes(24, 208), f32(1, 2), b)
    product = lambda b: hq.hq_fp8_linear(codes(8, 208), f32(2, 8), codes(24, 208), f32(1, 2), b)
    heads = lambda q, k, a, b: hq.hq_qk_norm_rope(q, k, a, b, f32(8, 32), f32(8, 32))
    x, b, q, k, w = (8, 200), (24,), (8, 4, 64), (8, 2, 64), (64,)
    for name, call in (
        ("x", lambda g: hq.hq_fp8_quantize_rows(fake(*x, grad=g))), ("x", lambda g: layer(fake(*x, grad=g), None)),
        ("bias", lambda g: layer(fake(*x), fake(*b, grad=g))), ("bias", lambda g: product(fake(*b, grad=g))),
        ("q", lambda g: heads(fake(*q, grad=g), fake(*k), None, None)), ("k", lambda g: heads(fake(*q), fake(*k, grad=g), None, None)),
        ("q_weight", lambda g: heads(fake(*q), fake(*k), fake(*w, grad=g), fake(*w))),
        ("k_weight", lambda g: heads(fake(*q), fake(*k), fake(*w), fake(*w, grad=g))),
    ):
        with pytest.raises(ValueError, match="^%s requires a gradient" % name):
            call(True)
        for grad, record in ((True, False), (False, True)):
            with torch.set_grad_enabled(record), pytest.raises(RuntimeError):
                call(grad)
    with pytest.raises(RuntimeError):
        hq.hq_fp8_quantize_blocks(fake(24, 200, grad=True))


def test_sizes_whose_products_wrap_are_refused(lib):
    """Counts of tiles and of heads beyond 64 bits."""
    for m, n in ((1 << 62, 1024), ((1 << 63) - 1, 16), (1 << 61, 128), ((1 << 63) - 1, 1), (1 << 40, 1)):
        assert lib.hq_fp8_linear(P, P, P, P, 0, None, m, n, 200, P, BF16, None) == UNSUPPORTED
        assert lib.hq_fp8_linear_kernel_name(I32, m, n, 200, BF16) == b"none"
    strides = (ctypes.c_int64 * 12)(*([512, 64] * 6))
    for t, heads in (((1 << 63) - 1, 4), (1 << 62, 4), (1 << 32, 1)):
        assert lib.hq_qk_norm_rope(P, P, F16, t, heads, 2, 64, strides, P, P, F16, P, P, 16, 64, 0, P, 8, 1e-6, P, P, None) == UNSUPPORTED
        assert lib.hq_qk_norm_rope_backward_workspace(F16, t, heads, 2, 64, 64) == 0
