"""The 4-bit key/value cache on the GPU: what append stores bit for bit, what read gives, attention against its definition in 64 bits.

The tolerance of attention is derived in kv4_reference.attention.  Codes of values that go in as they are (v; k without norm and rotation) are compared bit
for bit with the definition, decided in 64 bits, their scales with the same 32-bit steps in NumPy.  In test_norm_and_rotation codes of normalised, rotated keys may differ where the 64-bit value is close to a border:
a value of a head is off by (d / 2 + 12) 2^-24 of its pair's length (see test_gpu_qk.py), its transform by the sum of those over a block times
block^-1/2, with log2(block) + 3 roundings more."""
import numpy as np
import pytest
import torch

import paper_2512_05746_amd as hq
import kv4_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 0.0, "f32": 0.0}


def gpu(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def close(got, want, bound, dtype):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), "NaN in other places: %d, %d" % (np.isnan(got).sum(), nan.sum())
    off = np.where(nan, 0, np.abs(got - want))
    room = bound + HALF_STEP[dtype] * (np.abs(want) + bound) + TINY[dtype]
    room = np.where(nan, 1, room)
    worst = np.unravel_index(np.argmax(off - room), off.shape)
    assert (off <= room).all(), "%s: %g off, %g allowed, %d of %d" % (worst, off[worst], room[worst], (off > room).sum(), off.size)


class Call:
    """Sequences of the given new tokens and lengths in a cache of shuffled pages."""

    def __init__(self, new, lengths, kv_heads, d, page, seed=0, padding=0, content=True, spare=3, table_pages=None, had_block=None):
        rng = self.rng = np.random.default_rng(seed)
        self.new, self.lengths, self.page, self.d, self.kv_heads = list(new), list(lengths), page, d, kv_heads
        need = [max(0, -(-n // page)) for n in lengths]
        order = rng.permutation(sum(need) + spare)
        self.table = np.full((len(new), table_pages or max(max(need), 1)), -7, np.int32)
        at = 0
        for b, n in enumerate(need):
            m = min(n, self.table.shape[1])
            self.table[b, :m] = order[at:at + m]
            at += n
        self.begins = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.t = int(self.begins[-1]) + padding
        self.cache = ref.Cache(sum(need) + spare, kv_heads, page, d, rng if content else None)
        self.block = had_block or ref.block_of(d)
        self.on_gpu = hq.Kv4Cache(*(gpu(x) for x in self.cache.packed()), d, had_block)
        self.uniform = len(set(new)) == 1 and padding == 0

    def where(self, plain=False):
        return gpu(self.table), gpu(np.array(self.lengths, np.int32)), None if self.uniform and plain else gpu(self.begins)

    def places(self):
        """(sequence, place) of each token; -1, -1 of padding."""
        s, p = np.full(self.t, -1), np.full(self.t, -1)
        for b, (n, length) in enumerate(zip(self.new, self.lengths)):
            rows = np.arange(self.begins[b], self.begins[b + 1])
            s[rows], p[rows] = b, length - n + np.arange(n)
        return np.where(p < 0, -1, s), p

    def downloaded(self):
        return ref.Cache(self.cache.pages, self.kv_heads, self.page, self.d).unpack(*(x.cpu().numpy() for x in self.on_gpu[:4]))

    def check_attention(self, heads, dtype, window=0, sinks=0, scale=None, plain=False, spread=1.0, q=None, **kw):
        if q is None:
            q = self.rng.standard_normal((self.t, heads, self.d)) * spread
        q = gpu(q, DTYPES[dtype])
        got = hq.hq_kv4_attention(q, self.on_gpu, *self.where(plain), scale=scale, window=window, sinks=sinks, **kw)
        want, bound = ref.attention(q.double().cpu().numpy(), self.cache, self.table, self.lengths, self.begins,
                                    self.d ** -0.5 if scale is None else scale, window, sinks, self.block, dtype == "f32")
        close(got, want, bound, dtype)
        return got


# ---- attention ------------------------------------------------------------------------------------------------------------
RAGGED = ([1, 3, 0, 2, 1, 1, 5, 1], [1, 33, 17, 2, 0, 64, 131, 95])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,kv_heads,heads", [(8, 1, 1), (32, 2, 6), (40, 1, 4), (64, 2, 2), (72, 3, 3), (96, 2, 8), (128, 2, 8), (136, 1, 2), (160, 1, 3),
                                              (192, 2, 2), (224, 1, 5), (256, 1, 4)])
def test_heads_and_types(d, kv_heads, heads, dtype):
    Call(*RAGGED, kv_heads, d, 16, seed=d).check_attention(heads, dtype)


@pytest.mark.parametrize("page", [8, 16, 64, 256])
@pytest.mark.parametrize("heads", [1, 7, 16, 40])
def test_pages_and_groups(page, heads):
    Call([1, 2, 1, 4], [5, 130, 257, 31], 1, 64, page, seed=page + heads).check_attention(heads, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 2, 9, 16, 17, 40, 70, 129])
def test_new_tokens(new, dtype):
    """Rows for a key head from 2 to 258: every shape of workgroup."""
    Call([new, new, new], [new, new + 1, new + 77], 1, 64, 32, seed=new).check_attention(2, dtype, plain=True)


@pytest.mark.parametrize("d", [96, 200])
def test_many_rows_of_other_heads(d):
    call = Call([150, 1, 80, 33], [150, 20, 200, 33], 2, d, 16, seed=d, padding=5)
    assert not call.check_attention(2, "f16")[-5:].any()
    call.check_attention(6, "f32")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 0), (32, 4), (33, 40), (64, 1), (100, 64), (1000, 8), (1, 31)])
def test_window_and_sinks(window, sinks, dtype):
    call = Call([1, 3, 40, 2], [300, 131, 140, 33], 2, 64, 16, seed=window)
    call.check_attention(4, dtype, window=window, sinks=sinks)
    Call([90], [400], 1, 32, 8, seed=sinks).check_attention(1, dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1500, 70)])
@pytest.mark.parametrize("new,lengths", [([1], [5000]), ([1, 1, 1], [4097, 700, 1]), ([3, 1, 30], [2500, 3333, 1030]), ([70], [3000])])
def test_long_sequences_are_joined(new, lengths, window, sinks, dtype):
    Call(new, lengths, 2, 64, 64, seed=len(new)).check_attention(4, dtype, window=window, sinks=sinks, spread=2.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,kv_heads", [(80, 2), (96, 1), (128, 2), (160, 1), (200, 2), (256, 1)])
def test_parts_of_wide_heads(d, kv_heads, dtype):
    """Parts of few rows and of rows for more than one wave, heads that fill the lanes that own a row and heads that do not."""
    for new, lengths in (([1], [5000]), ([3, 1], [3333, 2100]), ([40], [3000])):
        Call(new, lengths, kv_heads, d, 64, seed=d).check_attention(kv_heads * 3, dtype, spread=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,kv_heads,heads", [(80, 8, 16), (32, 2, 6), (64, 3, 9), (128, 1, 12), (96, 5, 5), (160, 4, 8), (256, 2, 2)])
def test_parts_of_many_rows(d, kv_heads, heads, dtype):
    """Tokens times heads beyond 8192, in parts: heads that are and are not a multiple of those that a workgroup joins.  Some rows of each sequence
    against the definition."""
    rng = np.random.default_rng(d)
    most = 9000 // heads
    new = [int(n) for n in np.sort(rng.integers(20, most, 5))] + [most, 2]
    lengths = [n + int(m) for n, m in zip(new, rng.integers(0, 2500, 7))]
    lengths[2], lengths[6] = new[2] - 3, 1          # (rows that have no place)
    call = Call(new, lengths, kv_heads, d, 64, seed=d, padding=3)
    assert call.t * heads > 8192
    q = gpu(rng.standard_normal((call.t, heads, d)) * 2, DTYPES[dtype])
    got = hq.hq_kv4_attention(q, call.on_gpu, *call.where())
    assert not got[-3:].any()
    s, place = call.places()
    for b, (n, length) in enumerate(zip(new, lengths)):
        rows = np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, 2)]))
        for i in rows:
            at = int(call.begins[b]) + int(i)
            seen = length - n + int(i) + 1
            if seen <= 0:
                assert not got[at].any()
                continue
            want, bound = ref.attention(q[at:at + 1].double().cpu().numpy(), call.cache, call.table[b:b + 1], [seen], [0, 1], d ** -0.5, 0, 0, call.block,
                                        dtype == "f32")
            close(got[at:at + 1], want, bound, dtype)


def test_more_sequences_than_a_wave_has_lanes():
    rng = np.random.default_rng(3)
    lengths = rng.integers(0, 700, 150)
    lengths[[70, 140]] = 3000, 2100
    new = np.minimum(lengths, rng.integers(0, 3, 150))
    Call(new, lengths, 1, 32, 32, seed=5, padding=3).check_attention(2, "f32")


def test_scales():
    for scale in (0.0, -0.3, 1e-20, 2.0):
        Call([2, 1], [40, 9], 1, 64, 16).check_attention(2, "f32", scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,size,scale,keys", [(128, 1e-40, None, 1), (64, 3e-45, 1.0, 1), (64, 1e-3, 1e-38, 1), (64, 1e-7, 1e-20, 1), (96, 1e-6, 1e-45, 1), (256, 1.0, 3e-39, 1),
                                               (32, 1e-38, 1e-5, 1e31), (128, 1e-30, 0.1, 1e31), (64, 1e30, 1e-32, 1), (64, 1e30, 1e-20, 1e-10)])
def test_small_rows_and_scales(d, size, scale, keys, dtype):
    """Rows whose scores are next to nothing have the mean of what they see; lengths that leave the last tile of 32 with masked places."""
    if dtype == "f16":
        size, keys = min(max(size, 1e-7), 1e4), min(keys, 1.0)
    call = Call([3, 1, 2], [70, 33, 1025], 1, d, 16, seed=d)
    call.cache.ks *= np.float32(keys)
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), d)
    got = call.check_attention(2, dtype, scale=scale, spread=size)
    assert torch.isfinite(got).all()
    call.check_attention(2, dtype, scale=scale, spread=size, window=9, sinks=2)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("size", [1e-9, 1e4, 1e25])
def test_sizes_of_values(size, dtype):
    """Scales of v far from 1, and far from each other; rows of q far from 1."""
    if size > 1e20 and dtype == "f16":
        size = 1e3
    call = Call([2, 1, 3], [70, 33, 200], 1, 64, 16)
    call.cache.vs *= np.float32(size)
    call.cache.vs[::2] *= np.float32(1e-3)
    call.cache.ks *= np.float32(1e-6)
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    q = call.rng.standard_normal((call.t, 2, 64)) * (1e4 if dtype == "f16" else 1e6)
    q[0, 0] *= 1e-4
    q[1, 1] = 0
    if dtype == "f16" and size < 1e-6:
        call.cache.vs *= np.float32(1e5)
        call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    call.check_attention(2, dtype, q=q)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("size,other", [(1e36, 1), (1e36, 1e-36), (3e37, 1e-70), (1e-34, 1), (1e-34, 1e25), (1e-37, 1), (2e15, 1), (2e15, 1e-30), (1e-13, 1), (1e-13, 1e14)])
@pytest.mark.parametrize("lengths", [[70, 33, 200], [3000, 2500, 64]])
def test_ends_of_the_range_of_values(lengths, size, other, dtype):
    """Scales of v next to the ends of fp32, other pages another size, in one workgroup and in parts that are joined."""
    if dtype == "f16":      # (results are to be numbers of the type)
        size, other = (1e3, min(other, 1)) if size > 1 else (size, 1e3 / size if other > 1 else other)
    call = Call([2, 1, 3], lengths, 1, 64, 64)
    call.cache.vs *= np.float32(size)
    with np.errstate(under="ignore"):
        for b in range(3):
            call.cache.vs[call.table[b][call.table[b] >= 0][b % 2::2]] *= np.float32(other)
    call.cache.vs[:] = np.maximum(call.cache.vs, np.float32(2.0 ** -126))
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    call.check_attention(2, dtype)
    call.check_attention(2, dtype, window=100)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [3e3, 3e6, -1e8, 1e10, 1e20, 1e30])
def test_large_scores(scale, dtype):
    """Scores so large that a step of fp32 is many powers of two: nearly all of the weight on one token, which is not off by the other ones; one row of
    each call small, tokens in parts and in one workgroup, sizes of v that need all of the power of two next to scores."""
    for lengths, size in (([70, 33, 200], 1), ([3000, 2500, 64], 1), ([70, 300, 1400], 1e3 if dtype == "f16" else 1e30)):
        call = Call([2, 1, 3], lengths, 1, 64, 64, seed=int(np.log10(abs(scale))))
        call.cache.vs *= np.float32(size)
        for b, n in enumerate(lengths):          # a key whose score is apart from the others'
            place = n - 5
            call.cache.ks[call.table[b, place // 64], 0, place % 64] *= 8
        call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
        q = call.rng.standard_normal((call.t, 2, 64))
        q[1] *= 1e-7 if dtype == "f16" else 1e-30
        q = gpu(q, DTYPES[dtype])
        got = hq.hq_kv4_attention(q, call.on_gpu, *call.where(), scale=scale)
        assert torch.isfinite(got).all()
        q = q.cpu().double().numpy()
        with np.errstate(all="ignore"):
            want, bound = ref.attention(q, call.cache, call.table, call.lengths, call.begins, scale, 0, 0, call.block, dtype == "f32")
        if np.isfinite(bound[1]).all():     # (the small row; of large scores the bound knows nothing)
            close(got[1:2], want[1:2], bound[1:2], dtype)
        # where the largest score is far from the second: the value of that token
        apart = 0
        for row in (0, 2, 3, 4, 5):
            b = np.searchsorted(call.begins, row, side="right") - 1
            pos = call.lengths[b] - call.new[b] + row - call.begins[b]
            k, v = call.cache.rows(call.table[b], pos + 1)
            hq_row = ref.walsh(q[row], call.block) / 8
            for h in range(2):
                s = scale * (k[:, 0] @ hq_row[h])
                best = np.argsort(s)[-2:]
                if s[best[1]] - s[best[0]] > 200 + 1e-2 * abs(s[best[1]]):
                    want = ref.walsh(v[best[1], 0], call.block) / 8
                    off = np.abs(got[row, h].cpu().double().numpy() - want)
                    apart += 1
                    assert (off <= 2 * HALF_STEP["f16" if dtype != "bf16" else dtype] * (np.abs(want) + np.abs(v[best[1], 0]).sum())).all(), (row, h)
        assert apart


def test_peaked_rows():
    """Scores that differ by hundreds, the largest late, early and in the middle."""
    call = Call([1, 1, 1, 2], [300, 290, 64, 128], 1, 64, 16)
    for b, at in enumerate((299, 0, 40, 100)):
        call.cache.ks[call.table[b, at // 16], 0, at % 16] *= 100
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    for dtype in ("f16", "f32"):
        call.check_attention(2, dtype, spread=5.0)


def test_many_small_weights():
    """One token has the weight 1 and values of 0, 2000 others the weight 2^-15.3 (416.5 steps of a half below 2^-14, so that a half has it off by 1.2e-3):
    kept 2^6 times as large they are off by 2^-31 of the largest at most, which with the sums' 2000 x 2^-23 is a third of that."""
    call = Call([1], [2001], 1, 8, 16, content=False)
    cache = call.cache
    cache.k[..., 0], cache.v[...], cache.vs[...] = 2, 2, 1
    first = call.table[0, 0], 0, 0
    cache.ks[first], cache.v[first] = 1, 0
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in cache.packed()), 8)
    q = gpu(np.full((1, 1, 8), np.float32((24 - np.log2(416.5)) * np.log(2) / np.sqrt(8))), torch.float32)
    want, bound = ref.attention(q.double().cpu().numpy(), cache, call.table, call.lengths, call.begins, 1.0, 0, 0, call.block, True, 2.0 ** -31)
    assert (bound.max() < 5e-4 * np.abs(want).max())
    close(hq.hq_kv4_attention(q, call.on_gpu, *call.where(), scale=1.0), want, bound, "f32")


@pytest.mark.parametrize("seed", range(3))
def test_every_weight_by_itself(seed):
    """256 tokens whose values are a channel of their own each, so that the transformed result shows each weight; keys of one channel, so that scores
    are one product.  Errors counted, e of a score: the 8 sums and the halves of H q, 2^-22 each of sum |q| 8^-1/2; of the exponential's argument
    2^-22 (|s| + 16).  A weight: expm1(2 e), its two halves and the scale 2^-21, the sum of n weights n 2^-23 and 64 more for parts; a channel back
    through the transform 2^-20 of its block's largest.  A weight whose second half does not belong to the first is off by 2^-11 to 2^-10."""
    n, d, new, heads = 256, 256, 16, 16
    call = Call([new], [n], 1, d, 32, seed=seed, content=False, had_block=8)
    cache, where = call.cache, (call.table[0, np.arange(n) // 32], 0, np.arange(n) % 32)
    cache.k[where + (0,)], cache.v[where + (np.arange(n),)] = 2, 2
    cache.ks[where], cache.vs[where] = (np.exp(call.rng.normal(-1, 0.5, n)).astype(np.float32) for _ in "kv")
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in cache.packed()), d, 8)
    q = gpu(call.rng.standard_normal((new, heads, d)) * 2, torch.float32)
    got = hq.hq_kv4_attention(q, call.on_gpu, *call.where(), scale=1.0).cpu().double().numpy()
    q, ks, vs = q.cpu().double().numpy()[..., :8], cache.ks[where].astype(np.float64), cache.vs[where].astype(np.float64)
    s = q.sum(-1)[..., None] / np.sqrt(8) * ks
    s = np.where(np.arange(n) <= n - new + np.arange(new)[:, None, None], s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    want = p / p.sum(-1, keepdims=True) * vs
    e = np.abs(q).sum(-1)[..., None] / np.sqrt(8) * ks * 10 * 2.0 ** -22 + (np.where(p > 0, top - s, 0) + 16) * 2.0 ** -22
    grow = np.expm1(2 * e.max(-1, keepdims=True)) + 2.0 ** -21 + (n + 64) * 2.0 ** -23
    room = want * grow + 2.0 ** -20 * want.reshape(new, heads, -1, 8).max(-1).repeat(8, -1) + 2.0 ** -36 * vs.max()
    off = np.abs(ref.walsh(got, 8) / np.sqrt(8) - want)
    worst = np.unravel_index(np.argmax(off - room), off.shape)
    assert (off <= room).all(), "%s: %g off, %g allowed, of %g; %d" % (worst, off[worst], room[worst], want[worst], (off > room).sum())


def test_more_sequences_long_and_short():
    """Long ones come first, of every 64: of all lengths and orders, divided and not."""
    rng = np.random.default_rng(5)
    new = [int(x) for x in rng.integers(1, 40, 70)]
    lengths = [n + int(x) for n, x in zip(new, np.exp(rng.uniform(0, 7, 70)))]
    Call(new, lengths, 2, 32, 16, padding=3).check_attention(4, "f16")
    Call(new[:5], [n + 900 * (i % 2) for i, n in enumerate(lengths[:5])], 1, 32, 16).check_attention(2, "f32")


def test_on_another_device_than_the_current_one():
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    cache = hq.hq_kv4_cache(2, 16, 1, 32, device="cuda:1")
    one = torch.ones(1, dtype=torch.int32, device="cuda:1")
    with pytest.raises(ValueError, match="current device"):
        hq.hq_kv4_read(cache, one[:, None], one, 1)


def test_what_is_not_visible_is_not_looked_at():
    """NaN and infinities in slots behind the sequences' ends, in tokens outside the window, in other pages; entries of the table behind the last page."""
    call = Call([1, 2, 3], [45, 130, 91], 2, 64, 16, seed=9)
    args = dict(window=20, sinks=3)
    before = call.check_attention(4, "f32", **args)
    used = np.zeros(call.cache.ks.shape, bool)
    for b, (n, length) in enumerate(zip(call.new, call.lengths)):
        for pos in range(length - n, length):
            for j in range(pos + 1):
                if j > pos - 20 or j < 3:
                    used[call.table[b, j // 16], :, j % 16] = True
    for x in (call.cache.ks, call.cache.vs):
        x[~used] = call.rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38, 0], np.float32), (~used).sum())
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    q = np.random.default_rng(9)
    call.rng = np.random.default_rng(12)
    with np.errstate(all="ignore"):
        call.check_attention(4, "f32", **args)
        call.check_attention(4, "f16", **args)
    assert torch.isfinite(before).all()


def test_values_that_are_not_finite():
    """A NaN scale of a key or a value makes every row that sees it NaN, a row of q that is not finite itself only."""
    call = Call([4, 2], [50, 40], 1, 64, 16, seed=2)
    call.cache.ks[call.table[0, 47 // 16], 0, 47 % 16] = np.nan
    call.cache.vs[call.table[1, 39 // 16], 0, 39 % 16] = np.nan
    call.on_gpu = hq.Kv4Cache(*(gpu(x) for x in call.cache.packed()), 64)
    q = call.rng.standard_normal((call.t, 2, 64))
    q[0, 1, 5] = np.inf
    for dtype in ("f16", "f32"):
        got = call.check_attention(2, dtype, q=q)
        assert torch.isnan(got).all(-1).sum().item() == 1 + 2 * 3 + 2


def test_places_without_a_page():
    """Bad pages are NaN for the rows that see them, a length beyond the table for the whole sequence, a length below the new tokens leaves rows empty."""
    call = Call([3, 2, 2, 4], [40, 40, 30, 2], 1, 64, 16, seed=4)
    call.table[0, 2] = -1
    call.table[1, 0] = call.cache.pages
    call.lengths[2] = 49     # three pages of 16
    call.lengths[3] = 2
    for dtype in ("f16", "f32"):
        got = call.check_attention(2, dtype)
        assert torch.isnan(got[:7]).all() and not got[7:9].any() and torch.isfinite(got).sum() == 4 * 2 * 64
    call.lengths[3] = -5
    assert not call.check_attention(2, "f32")[7:].any()
    call.check_attention(2, "f32", window=3)


def test_views_results_streams():
    call = Call([1, 1, 1, 1], [40, 700, 33, 8], 2, 64, 16)
    rows = gpu(call.rng.standard_normal((4, 12 * 64)), torch.float16)
    q = rows[:, :256].view(4, 4, 64)
    want = hq.hq_kv4_attention(q.contiguous(), call.on_gpu, *call.where())
    assert torch.equal(hq.hq_kv4_attention(q, call.on_gpu, *call.where()), want)
    out = torch.full((4, 3, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    got = hq.hq_kv4_attention(q, call.on_gpu, *call.where(plain=True), out=out[:, 1])
    assert got.data_ptr() == out[:, 1].data_ptr() and torch.equal(out[:, 1], want)
    assert (out[:, 0] == 7).all() and (out[:, 2] == 7).all()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(1000000)
        late = hq.hq_kv4_attention(q, call.on_gpu, *call.where())
        torch.cuda.current_stream().synchronize()
    assert torch.equal(late, want)
    assert hq.hq_kv4_attention(q[:0], call.on_gpu, *call.where()[:2], torch.zeros(5, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)


@pytest.mark.parametrize("lengths", [[40, 300], [3000, 5000]])
def test_graph_of_growing_sequences(lengths):
    """One captured step, replayed as the sequences grow, against eager calls; two graphs share a pool of memory, and eager work runs between."""
    call = Call([1, 1], [n + 8 for n in lengths], 2, 64, 16, content=False)
    d, q = 64, torch.randn(2, 4, 64, device="cuda", dtype=torch.float16)
    k, v = (torch.randn(2, 2, 64, device="cuda", dtype=torch.float16) for _ in "kv")
    cos, sin = torch.rand(8192, 32, device="cuda"), torch.rand(8192, 32, device="cuda")
    table = gpu(call.table)
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    filled = hq.Kv4Cache(*(gpu(x) for x in ref.Cache(call.cache.pages, 2, 16, 64, np.random.default_rng(0)).packed()), 64)
    eager = hq.Kv4Cache(*(x.clone() for x in filled[:4]), 64)

    def step(cache):
        turned = hq.hq_kv4_append(q, k, v, None, None, cos, sin, cache, table, length)
        return hq.hq_kv4_attention(turned, cache, table, length)

    step(hq.Kv4Cache(*(x.clone() for x in filled[:4]), 64))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for window in (0, 100):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0].pool() if graphs else None):
            outs.append(step(filled) if window == 0 else hq.hq_kv4_attention(q, filled, table, length, window=window))
        graphs.append(g)
    for turn in range(6):
        for x in (q, k, v):
            x.normal_()
        graphs[0].replay()
        first = outs[0].clone()
        graphs[1].replay()
        assert torch.equal(first, step(eager)), turn
        assert torch.equal(outs[1], hq.hq_kv4_attention(q, eager, table, length, window=100)), turn
        assert all(torch.equal(a, b) for a, b in zip(filled[:4], eager[:4]))
        torch.cuda.synchronize()
        length += 1


def test_far_pages():
    """Codes beyond 4 GiB and scales: the same sequence in the first and in the last pages of a long cache."""
    page, heads, d = 256, 8, 256
    pages = (5 << 30) // (page * heads * d // 2)
    small = Call([1, 2], [1000, 513], heads, d, page, seed=1, spare=0)
    big = hq.hq_kv4_cache(pages, page, heads, d)
    for to, x in zip(big[:4], small.on_gpu[:4]):
        to[-x.shape[0]:] = x
    q = torch.randn(3, 16, d, device="cuda", dtype=torch.bfloat16)
    table, lengths, begins = small.where()
    far = table + (pages - small.cache.pages)
    assert torch.equal(hq.hq_kv4_attention(q, big, far, lengths, begins), hq.hq_kv4_attention(q, small.on_gpu, table, lengths, begins))
    for a, b in zip(hq.hq_kv4_read(big, far, lengths, 3, begins), hq.hq_kv4_read(small.on_gpu, table, lengths, 3, begins)):
        assert torch.equal(a, b)
    new = [torch.randn(3, h, d, device="cuda", dtype=torch.bfloat16) for h in (16, heads, heads)]
    none = torch.zeros(1, 0, device="cuda")
    for cache, where in ((big, far), (small.on_gpu, table)):
        hq.hq_kv4_append(*new, None, None, none, none, cache, where, lengths, begins, eps=None)
    for x, y in zip(big[:4], small.on_gpu[:4]):
        assert torch.equal(x[-y.shape[0]:], y) and not x[:-y.shape[0]].any()


# ---- append and read ------------------------------------------------------------------------------------------------------
def append(call, heads, dtype, rotary=0, norm=False, interleaved=False, positions=None, weights="same", x=None, table=None, strided=True, **kw):
    """(the queries, inputs) of one append; x: q, k, v as arrays."""
    rng, hk, d = call.rng, call.kv_heads, call.d
    dt = DTYPES[dtype]
    if x is None:
        x = [rng.standard_normal((call.t, h, d)) * 2 for h in (heads, hk, hk)]
    if strided:
        whole = gpu(np.concatenate(x, 1), dt)
        q, k, v = whole[:, :heads], whole[:, heads:heads + hk], whole[:, heads + hk:]
    else:
        q, k, v = (gpu(y, dt) for y in x)
    w = (None, None)
    if norm and weights != "none":
        w = tuple(gpu(1 + 0.2 * rng.standard_normal(d), torch.float32 if weights == "f32" else dt) for _ in "qk")
    table = table or max([n for n in call.lengths] + [1]) + 1
    angle = np.outer(np.arange(table), 10000.0 ** (-np.arange(0, rotary, 2) / max(rotary, 1)))
    cos, sin = gpu(np.cos(angle).astype(np.float32)), gpu(np.sin(angle).astype(np.float32))
    got = hq.hq_kv4_append(q, k, v, *w, cos, sin, call.on_gpu, *call.where(), positions=None if positions is None else gpu(positions),
                           eps=1e-6 if norm else None, interleaved=interleaved, **kw)
    return got, (q, k, v, w, cos.cpu().double().numpy(), sin.cpu().double().numpy())


def turned(x, w, cos, sin, place, rotary, norm, interleaved):
    """(heads in 64 bits, how far fp32 may be off), [t, heads, d]; place < 0: zeros, beyond the tables NaN"""
    x = x.double().cpu().numpy()
    d = x.shape[-1]
    n = x
    if norm:
        n = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * (1 if w is None else w.double().cpu().numpy())
    at = np.clip(place, 0, len(cos) - 1)
    c, s = cos[at][:, None], sin[at][:, None]
    first = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    a, b = n[..., first[0]], n[..., first[1]]
    y, size = n.copy(), np.abs(n)
    y[..., first[0]], y[..., first[1]] = a * c - b * s, b * c + a * s
    size[..., first[0]] = size[..., first[1]] = np.sqrt(a * a + b * b)
    y = np.where((place < 0)[:, None, None], 0, np.where((place >= len(cos))[:, None, None], np.nan, y))
    return y, size * (d / 2 + 12) * 2.0 ** -24


def check_codes(call, after, before, which, want_codes, want_scale, sure, scale_room=0.0):
    """The slots of the call's tokens hold want_codes where `sure`, their neighbours of 4 bits elsewhere; all other slots what they held."""
    s, place = call.places()
    codes, scales = (after.k, after.ks) if which == "k" else (after.v, after.vs)
    old, old_scales = (before.k, before.ks) if which == "k" else (before.v, before.vs)
    touched = np.zeros(scales.shape, bool)
    differ = 0
    for row in range(call.t):
        if place[row] < 0 or (column := place[row] // call.page) >= call.table.shape[1]:
            continue
        page = call.table[s[row], column]
        if page < 0 or page >= call.cache.pages:
            continue
        at = (page, slice(None), place[row] % call.page)
        touched[at] = True
        got, want = codes[at], want_codes[row]
        bad = (got != want) & ~((got & 7 == 0) & (want & 7 == 0))      # (a zero of either sign)
        assert not (bad & sure[row]).any(), (which, row, np.argwhere(bad & sure[row])[:3], got[bad], want[bad])
        differ += bad.sum()
        assert (np.abs(ref.VALUES[got[bad]] - ref.VALUES[want[bad]]) <= 2).all()
        nan = np.isnan(want_scale[row])
        assert (np.isnan(scales[at]) == nan).all()
        assert (np.abs(scales[at] - want_scale[row])[~nan] <= scale_room * np.abs(want_scale[row])[~nan]).all()
    assert np.array_equal(codes[~touched], old[~touched])
    assert np.array_equal(scales[~touched].view(np.int32), old_scales[~touched].view(np.int32))
    return differ


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,had_block", [(8, None), (32, None), (32, 4), (40, 1), (64, None), (72, 2), (80, None), (96, None), (128, None), (128, 64), (160, None),
                                         (192, 16), (256, None)])
def test_stored_bit_for_bit(d, had_block, dtype):
    """v, and k that is neither normalised nor rotated: the documented 32-bit steps."""
    call = Call([1, 9, 0, 30, 2, 8], [1, 20, 5, 41, 64, 16], 3, d, 16, seed=d, padding=3, had_block=had_block)
    before = call.downloaded()
    got, (q, k, v, _, _, _) = append(call, 6, dtype)
    after = call.downloaded()
    for which, x in (("k", k), ("v", v)):
        codes, scale = ref.encode(ref.transformed(x.float().cpu().numpy(), call.block))
        check_codes(call, after, before, which, codes, scale, np.ones(codes.shape, bool))
    assert torch.equal(got[:-3], q[:-3]) and not got[-3:].any()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,rotary,interleaved,norm,weights", [(64, 64, False, True, "same"), (128, 128, False, True, "f32"), (80, 40, True, False, "none"),
                                                                (72, 72, False, True, "same"), (96, 36, False, True, "none"), (40, 10, False, False, "none"),
                                                                (256, 128, False, True, "f32"), (32, 6, True, True, "same"), (160, 160, True, True, "same")])
def test_norm_and_rotation(d, rotary, interleaved, norm, weights, dtype):
    call = Call([1, 9, 30, 2], [1, 20, 41, 64], 2, d, 16, seed=d + rotary, padding=2)
    before = call.downloaded()
    got, (q, k, v, w, cos, sin) = append(call, 6, dtype, rotary, norm, interleaved, weights=weights)
    _, place = call.places()
    close(got, *turned(q, w[0], cos, sin, place, rotary, norm, interleaved), dtype)
    y, off = turned(k, w[1], cos, sin, place, rotary, norm, interleaved)
    z = ref.walsh(y, call.block) / np.sqrt(call.block)
    z_off = (np.abs(ref.walsh(np.eye(d), call.block)) / np.sqrt(call.block) @ off[..., None])[..., 0] + \
        (np.abs(ref.walsh(np.eye(d), call.block)) / np.sqrt(call.block) @ np.abs(y)[..., None])[..., 0] * (call.block.bit_length() + 3) * 2.0 ** -24
    top = np.abs(z).max(-1, keepdims=True)
    scale = np.where(top > 0, top / 6, 1)
    t, t_off = z / scale, z_off / scale + np.abs(z / scale) * (z_off.max(-1, keepdims=True) / scale / 6 + 2.0 ** -22)
    sure = (np.abs(np.abs(t)[..., None] - ref.BORDERS) > t_off[..., None]).all(-1)
    assert sure.mean() > 0.99
    room = np.max(z_off.max(-1, keepdims=True)[place >= 0] / top[place >= 0]) + 2.0 ** -22
    differ = check_codes(call, call.downloaded(), before, "k", ref.codes_of(t), scale[..., 0], sure, room)
    assert differ <= (~sure).sum()
    codes, scale = ref.encode(ref.transformed(v.float().cpu().numpy(), call.block))
    check_codes(call, call.downloaded(), before, "v", codes, scale, np.ones(codes.shape, bool))


def stored_codes(call, which, row):
    """The codes that the cache holds for a row of the call."""
    after = call.downloaded()
    s, place = call.places()
    codes = after.k if which == "k" else after.v
    return np.stack([codes[call.table[s[r], place[r] // call.page], :, place[r] % call.page] for r in row])


# (a, b) of which sums are a + b and a - b: 6 (a - b) / (a + b) is a border, and nothing of it needs more than 6 bits
TIES = {0.25: (25, 23), 0.75: (9, 7), 1.25: (29, 19), 1.75: (31, 17), 2.5: (17, 7), 3.5: (19, 5), 5.0: (11, 1)}


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,had_block", [(8, 2), (64, None), (128, None), (128, 32), (72, None), (160, None), (256, None)])
def test_ties_go_to_even(d, had_block, dtype, norm):
    """Two channels of a block, so that every sum of it is the largest or a border's number of times a sixth of it, exactly; at sizes for which scales have
    all kinds of roundings, and one step of fp32 to either side.  The norm's factor is the same for all of a head."""
    call = Call([9, 33, 14], [9, 40, 30], 7, d, 16, seed=d, had_block=had_block)
    rng, block = call.rng, call.block
    x = [np.zeros((call.t, h, d), np.float32) for h in (7, 7, 7)]
    for y in x[1:]:
        for row in range(call.t):
            for h, border in enumerate(TIES):
                pair, at = np.array(TIES[border], np.float32), rng.integers(d // block) * block + rng.choice(block, 2, replace=False)
                pair *= rng.choice([-1, 1], 2) * 2.0 ** rng.integers(-4, 4)
                if dtype == "f32" and row % 3 == 1:     # nearly a tie
                    pair[1] = np.nextafter(pair[1], pair[1] * rng.choice([0, 2]), dtype=np.float32)
                if dtype == "f32" and row % 3 == 2:     # a tie at any size
                    pair *= np.float32(rng.integers(1, 1 << 18))
                y[row, h, at] = pair
    before = call.downloaded()
    _, (q, k, v, w, _, _) = append(call, 7, dtype, norm=norm, weights="none", x=x)
    after, sure = call.downloaded(), np.ones((call.t, 7, d), bool)
    for which, y in (("v", v), ("k", k)):
        assert torch.equal(y.float().cpu(), torch.from_numpy(x[2 if which == "v" else 1]))
        z = ref.transformed(y.float().cpu().numpy(), block)
        codes, scale = ref.encode(z)
        ratio = 6 * np.abs(z[0]) / np.abs(z[0]).max(-1, keepdims=True)
        tied = (np.abs(ratio[..., None] - np.array(list(TIES))) < 1e-12).any(-1)
        assert tied[::3].any(-1).all() and (codes[tied] % 2 == 0).all()
        if which == "k" and norm:   # (codes do not depend on the factor; scales are those of normalised heads, off by fp32 steps)
            n = (y.double() * torch.rsqrt(y.double().square().mean(-1, keepdim=True) + 1e-6)).cpu().numpy()
            scale = np.abs(ref.walsh(n, block)).max(-1) * block ** -0.5 / 6
            check_codes(call, after, before, which, codes, scale, sure, (d / 2 + 24) * 2.0 ** -24)
        else:
            check_codes(call, after, before, which, codes, scale, sure)


@pytest.mark.parametrize("dtype,size", [("f16", 1), ("bf16", 1), ("f32", 1), ("f32", 1e-37), ("f32", 1e-39), ("bf16", 1e-38), ("f32", 1e30)])
def test_codes_of_many_heads(dtype, size):
    """Values: every code is that of the definition, next to the least scale too."""
    call = Call([1500, 1500], [1500, 1501], 8, 128, 64, seed=3, content=False)
    x = [call.rng.standard_normal((call.t, 8, 128)).astype(np.float32) * np.float32(size) for _ in "qkv"]
    x[2][:, ::2] *= np.exp(2 * call.rng.standard_normal((call.t, 4, 128))).astype(np.float32)
    _, (q, k, v, *_) = append(call, 8, dtype, x=x, weights="none", table=1)
    for which, y in (("k", k), ("v", v)):
        want, scale = ref.encode(ref.transformed(y.float().cpu().numpy(), call.block))
        got = stored_codes(call, which, range(call.t))
        bad = (got != want) & ~((got & 7 == 0) & (want & 7 == 0))
        assert np.isfinite(scale).all() and not bad.any(), (which, bad.sum(), np.argwhere(bad)[:3])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,rotary,interleaved,norm,weights", [(128, 128, False, True, "same"), (128, 64, False, True, "f32"), (64, 64, True, True, "none"),
                                                                (80, 72, False, False, "none"), (160, 20, False, True, "f32"), (32, 32, False, True, "same"),
                                                                (256, 256, False, True, "same"), (192, 32, False, False, "none"), (128, 16, False, False, "none")])
def test_codes_of_turned_keys(d, rotary, interleaved, norm, weights, dtype):
    """Keys that are normalised and turned: every code is that of the definition in 64 bits, but next to a border by less than what 64-bit steps are off:
    2^-53 for each of 3 (log2(block) + 4) and a number up to 6, of sums that are up to a head's length in size, 2^-40 with room."""
    rows = 600000 // d
    call = Call([rows, rows], [rows, rows + 5], 2, d, 64, seed=d + rotary, content=False)
    _, (q, k, v, w, cos, sin) = append(call, 2, dtype, rotary, norm, interleaved, weights=weights)
    y, _ = turned(k, w[1], cos, sin, call.places()[1], rotary, norm, interleaved)
    sums = ref.walsh(y, call.block)
    t = 6 * np.abs(sums) / np.abs(sums).max(-1, keepdims=True)
    sure = (np.abs(t[..., None] - ref.BORDERS) > 2.0 ** -40).all(-1)
    assert sure.mean() > 0.999999
    got, want = stored_codes(call, "k", range(call.t)), ref.exact_codes(sums)
    bad = (got != want) & ~((got & 7 == 0) & (want & 7 == 0)) & sure
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3])


def test_ties_of_many_heads():
    """40 heads one after the other in a lane: ties in the first ones and the last."""
    t, heads, d = 17000, 40, 136
    call = Call([t], [t], heads, d, 256, content=False)
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((t, heads, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in "kv")
    rows = np.sort(call.rng.choice(t, 200, replace=False))
    for x in (k, v):
        some = np.zeros((len(rows), heads, d), np.float32)
        for i in range(len(rows)):
            for h in range(heads):
                at = call.rng.integers(d // 8) * 8 + call.rng.choice(8, 2, replace=False)
                some[i, h, at] = np.array(list(TIES.values())[call.rng.integers(7)], np.float32) * call.rng.choice([-1, 1], 2)
        x[torch.from_numpy(rows).cuda()] = gpu(some, torch.bfloat16)
    none = torch.zeros(1, 0, device="cuda")
    hq.hq_kv4_append(torch.zeros_like(k), k, v, None, None, none, none, call.on_gpu, *call.where(), eps=None)
    for which, x in (("k", k), ("v", v)):
        x = x[torch.from_numpy(rows).cuda()].float().cpu().numpy()
        got, (want, _) = stored_codes(call, which, rows), ref.encode(ref.transformed(x, call.block))
        bad = (got != want) & ~((got & 7 == 0) & (want & 7 == 0))
        assert not bad.any(), (which, bad.sum(), np.argwhere(bad)[:3])


@pytest.mark.parametrize("page", [8, 32])
def test_one_by_one_is_all_at_once(page):
    """Tokens that come one at a time, in pieces and at once leave the same bits, whatever was in the pages."""
    d, hk, total = 64, 2, 45
    x = [np.random.default_rng(1).standard_normal((total, h, d)) for h in (4, hk, hk)]
    kept = []
    for cuts in ([45], [1] * 45, [7, 1, 1, 15, 8, 13], [40, 5]):
        call = Call([45], [45], hk, d, page, seed=6)
        at, rows = 0, []
        for n in cuts:
            call.new, call.lengths, call.t, call.begins = [n], [at + n], n, np.array([0, n], np.int32)
            rows.append(append(call, 4, "f16", 64, True, x=[y[at:at + n] for y in x], weights="none", table=64)[0])
            at += n
        kept.append(list(call.on_gpu[:4]) + [torch.cat(rows)])
    for other in kept[1:]:
        for a, b in zip(kept[0], other):
            assert torch.equal(a, b)


def test_padding_and_positions():
    """Explicit positions: negative ones are padding, ones beyond the tables NaN (their values are stored); lengths below the new tokens."""
    call = Call([3, 12, 4], [20, 40, 2], 2, 64, 16, seed=8, padding=1)
    positions = np.array([5, -1, 100] + list(range(9, 21)) + [1, 2, 3, 4] + [0], np.int64)
    for dt in (np.int64, np.int32):
        before = call.downloaded()
        got, (q, k, v, w, cos, sin) = append(call, 4, "f32", 64, True, positions=positions.astype(dt), table=60)
        s, place = call.places()
        place = np.where(positions < 0, -1, place)
        angle = np.where(place < 0, -1, positions)
        close(got, *turned(q, w[0], cos, sin, angle, 64, True, False), "f32")
        assert torch.isnan(got[2]).all() and not got[1].any() and not got[15:17].any() and not got[-1].any()
        after = call.downloaded()
        call.places = lambda: (s, place)
        codes, scale = ref.encode(ref.transformed(v.float().cpu().numpy(), 64))
        check_codes(call, after, before, "v", codes, scale, np.ones(codes.shape, bool))
        assert np.isnan(after.ks[call.table[0, 1], :, 19 % 16]).all() and not after.k[call.table[0, 1], :, 19 % 16].any()
        del call.places


def test_places_without_a_page_are_not_written():
    call = Call([20, 5, 3], [40, 40, 30], 1, 64, 16, seed=4)
    call.table[0, 1] = -1
    call.table[1, 2] = call.cache.pages
    call.lengths[2] = 50     # places 47, 48, 49, the table has three columns of 16
    before = call.downloaded()
    got, (q, k, v, _, _, _) = append(call, 2, "f16")
    assert torch.equal(got, q)
    codes, scale = ref.encode(ref.transformed(v.float().cpu().numpy(), 64))
    check_codes(call, call.downloaded(), before, "v", codes, scale, np.ones(codes.shape, bool))
    k_read, v_read = hq.hq_kv4_read(call.on_gpu, *call.where()[:2], call.t, call.where()[2], y_dtype=torch.float32)
    s, place = call.places()
    gone = np.array([place[r] // 16 >= 3 or not 0 <= call.table[s[r], place[r] // 16] < call.cache.pages for r in range(call.t)])
    assert gone.sum() == 12 + 5 + 3   # (place 47 is in the third column, which a sequence of 30 tokens left at -7)
    assert (torch.isnan(k_read).all(-1).all(-1).cpu().numpy() == gone).all() and (torch.isnan(v_read).all(-1).all(-1).cpu().numpy() == gone).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_values_that_are_not_finite_are_stored_as_nan(dtype):
    call = Call([6], [22], 2, 64, 16, seed=4)
    x = [call.rng.standard_normal((6, h, 64)) for h in (2, 2, 2)]
    x[1][1, 0, 3], x[2][2, 1, 9], x[1][4, 1], x[2][4, 1] = np.inf, np.nan, 0, 0
    before = call.downloaded()
    append(call, 2, dtype, x=x)
    after = call.downloaded()
    for which, y in (("k", x[1]), ("v", x[2])):
        codes, scale = ref.encode(ref.transformed(gpu(y, DTYPES[dtype]).float().cpu().numpy(), 64))
        assert np.isnan(scale).sum() == 1 and (scale == 1).sum() == 1
        check_codes(call, after, before, which, codes, scale, np.ones(codes.shape, bool))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d,had_block", [(8, None), (32, None), (40, 1), (72, 2), (96, None), (128, None), (128, 32), (192, None), (256, None)])
def test_read(d, had_block, dtype):
    """Sums of codes are exact in fp32; then come one product with scale x factor, bit for bit, and the type's rounding.  (A multiplication whose result is
    wanted in 16 bits may be one instruction that rounds once: that and rounding twice are both within half a step of 16 bits and one of fp32.)"""
    lengths = [1, 20, 0, 41, 64, 7]
    for new in (lengths, [1, 3, 0, 40, 9, 7]):
        call = Call(new, lengths, 3, d, 16, seed=d, padding=4, had_block=had_block)
        k, v = hq.hq_kv4_read(call.on_gpu, *call.where()[:2], call.t, call.where()[2], y_dtype=DTYPES[dtype])
        s, place = call.places()
        for got, codes, scales in ((k, call.cache.k, call.cache.ks), (v, call.cache.v, call.cache.vs)):
            want = np.zeros((call.t, 3, d), np.float32)
            for row in range(call.t):
                if place[row] >= 0:
                    at = (call.table[s[row], place[row] // 16], slice(None), place[row] % 16)
                    want[row] = ref.walsh(ref.VALUES[codes[at]].astype(np.float32), call.block) * (scales[at] * ref.factor(call.block))[:, None]
            if dtype == "f32":
                assert torch.equal(got, gpu(want))
            close(got, want.astype(np.float64), 2.0 ** -24 * np.abs(want), dtype)


def test_read_uniform_and_out():
    call = Call([4, 4], [20, 9], 2, 64, 16)
    a = hq.hq_kv4_read(call.on_gpu, *call.where()[:2], 8)
    out = (torch.empty(8, 2, 64, dtype=torch.float16, device="cuda"), torch.empty(8, 2, 64, dtype=torch.float16, device="cuda"))
    b = hq.hq_kv4_read(call.on_gpu, *call.where()[:2], 8, call.where()[2], out=out)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and b[0].data_ptr() == out[0].data_ptr()


def test_append_in_place_on_another_stream():
    call = Call([3, 2], [20, 9], 2, 64, 16, seed=3)
    other = Call([3, 2], [20, 9], 2, 64, 16, seed=3)
    want, (q, k, v, w, cos, sin) = append(call, 4, "f16", 64, True)
    with torch.cuda.stream(torch.cuda.Stream()):
        got, (q2, *_) = append(other, 4, "f16", 64, True, out=None)
        torch.cuda.current_stream().synchronize()
    assert torch.equal(got, want)
    same = hq.hq_kv4_append(q, k, v, *w, gpu(cos.astype(np.float32)), gpu(sin.astype(np.float32)), call.on_gpu, *call.where(), out=q)
    assert same.data_ptr() == q.data_ptr() and torch.equal(same, want)
    assert all(torch.equal(a, b) for a, b in zip(call.on_gpu[:4], other.on_gpu[:4]))


# ---- together -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_block_served_token_by_token(dtype):
    """Projection in 8-bit floats, append, attention: a prompt in two chunks and single tokens, against attention over the numbers that read gives."""
    dt, heads, hk, d, width, page = DTYPES[dtype], 8, 2, 64, 256, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    wq, sw = hq.hq_fp8_quantize_blocks(rand((heads + 2 * hk) * d, width) * width ** -0.5)
    norm = [(1 + 0.1 * rand(d)).to(dt) for _ in "qk"]
    angle = torch.outer(torch.arange(300.0), 10000.0 ** (-torch.arange(0, d, 2) / d)).cuda()
    cache = hq.hq_kv4_cache(64, page, hk, d)
    table = torch.randperm(64, generator=gen, device="cuda")[:60].int().view(3, 20)
    length = torch.zeros(3, dtype=torch.int32, device="cuda")
    for new in ([100, 3, 0], [40, 1, 200], [1, 1, 1], [1, 1, 1], [2, 5, 1]):
        n = torch.tensor(new, dtype=torch.int32, device="cuda")
        begins = torch.cat([n.new_zeros(1), n.cumsum(0).int()])
        length = length + n
        t = sum(new)
        qkv = hq.hq_act_quant_fp8_linear(rand(t, width).to(dt), wq, sw, y_dtype=dt).view(t, -1, d)
        q = hq.hq_kv4_append(qkv[:, :heads], qkv[:, heads:heads + hk], qkv[:, heads + hk:], *norm, angle.cos(), angle.sin(), cache, table, length, begins)
        got = hq.hq_kv4_attention(q, cache, table, length, begins).double().cpu()
        total = int(length.sum())
        ends = torch.cat([n.new_zeros(1), length.cumsum(0).int()])
        k, v = (x.double().cpu() for x in hq.hq_kv4_read(cache, table, length, total, ends, y_dtype=torch.float32))
        qd, at = q.double().cpu(), 0
        for b in range(3):
            m, size = new[b], int(length[b])
            lo = int(ends[b])
            kk, vv = (x[lo:lo + size].repeat_interleave(heads // hk, 1) for x in (k, v))
            s = torch.einsum("ihd,jhd->hij", qd[at:at + m], kk) * d ** -0.5
            s = s.masked_fill(torch.arange(size)[None] > torch.arange(size - m, size)[:, None], -np.inf)
            want = torch.einsum("hij,jhd->ihd", s.softmax(-1), vv)
            # scores of these norms are below 64 x 1.3^2 / 8 = 14 in size: H q off by 2^-11 of 14 changes a weight by 0.7 % at most, twice
            assert m == 0 or (got[at:at + m] - want).norm() <= 0.016 * want.norm()
            at += m
