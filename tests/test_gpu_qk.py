"""Norm and rotation of query and key heads, and their gradients, against the definition in 64 bits (NumPy).

Tolerances: a result is a few fp32 products of values of its own pair after one sum over the head; every term is non-negative in that sum, so it is off
by at most (d + 4) 2^-24 of itself (whatever its order) and its root by half of that; cosine, sine and weights are given.  A result is then off by
at most (d / 2 + 10) 2^-24 of the length of its pair (a, b), plus the rounding to its type.  Gradients: the projection is a sum of d terms of either
sign, bounded in the same way by the sum of their magnitudes.  Sums for the weights have tokens x heads terms."""
import numpy as np
import pytest
import torch

import paper_2512_05746_amd as hq

pytestmark = pytest.mark.gpu

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 0.0, "f32": 0.0}
EPS = 1e-6


def tables(positions, rotary):
    angle = np.outer(np.arange(positions), 10000.0 ** (-np.arange(0, rotary, 2) / max(rotary, 1)))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def pairs(v, r, interleaved):
    return (v[..., 0:r:2], v[..., 1:r:2]) if interleaved else (v[..., :r // 2], v[..., r // 2:r])


def joined(a, b, rest, interleaved):
    turned = np.stack([a, b], -1).reshape(a.shape[:-1] + (-1,)) if interleaved else np.concatenate([a, b], -1)
    return np.concatenate([turned, rest], -1)


def turned(v, cos, sin, r, interleaved):
    a, b = pairs(v, r, interleaved)
    return joined(a * cos - b * sin, b * cos + a * sin, v[..., r:], interleaved)


def pair_length(v, r, interleaved):
    a, b = pairs(v, r, interleaved)
    size = np.sqrt(a * a + b * b)
    return joined(size, size, np.abs(v[..., r:]), interleaved)


def reference(x, w, cos, sin, pos, r, interleaved, dy=None, eps=EPS):
    """(y, bound) or ((dx, bound), (dw, bound)) without roundings to the type."""
    x, w, d = x.astype(np.float64), w.astype(np.float64), x.shape[-1]
    live = (pos >= 0)[:, None, None]
    c, s = (t.astype(np.float64)[np.maximum(pos, 0)][:, None] for t in (cos, sin))
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    unit = x * rstd
    rel = (d / 2 + 10) * 2.0 ** -24
    if dy is None:
        n = unit * w
        return np.where(live, turned(n, c, s, r, interleaved), 0), np.where(live, pair_length(n, r, interleaved), 0) * rel
    g = np.where(live, turned(dy.astype(np.float64), c, -s, r, interleaved), 0)
    size = np.where(live, pair_length(dy.astype(np.float64), r, interleaved), 0)
    dw, dw_bound = (g * unit).sum((0, 1)), (size * np.abs(unit)).sum((0, 1)) * (rel + x.shape[0] * x.shape[1] * 2.0 ** -24)
    gw = g * w
    dot = (gw * unit).mean(-1, keepdims=True)
    most = (size * np.abs(w * unit)).mean(-1, keepdims=True)
    dx = rstd * (gw - unit * dot)
    bound = rstd * (size * np.abs(w) + np.abs(unit) * most) * (2 * d + 20) * 2.0 ** -24
    return (dx, bound), (dw, dw_bound)


def close(got, want, bound, dtype):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape
    off, room = np.abs(got - want), bound + ULP[dtype] * (np.abs(want) + bound) + TINY[dtype]
    worst = np.unravel_index(np.argmax(off - room), off.shape)
    assert (off <= room).all(), "%s: %g off, %g allowed" % (worst, off[worst], room[worst])


class Case:
    def __init__(self, t, heads, kv_heads, d, rotary, dtype, interleaved=False, weights="same", seed=0, pos="index", table=64):
        rng = np.random.default_rng(seed + t * 7 + d)
        dt = DTYPES[dtype]
        self.dtype, self.r, self.interleaved = dtype, rotary, interleaved
        qkv = torch.from_numpy((rng.standard_normal((t, (heads + 2 * kv_heads) * d)) * 2).astype(np.float32)).to(dt).cuda()
        self.q = qkv[:, :heads * d].view(t, heads, d)
        self.k = qkv[:, heads * d:(heads + kv_heads) * d].view(t, kv_heads, d)
        w = lambda: torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)).to(torch.float32 if weights == "f32" else dt).cuda()
        self.wq, self.wk = (None, None) if weights == "none" else (w(), w())
        grad = lambda h: torch.from_numpy(rng.standard_normal((t, h, d)).astype(np.float32)).to(dt).cuda()
        self.dq, self.dk = grad(heads), grad(kv_heads)
        table = max(table, t if pos == "index" else 1)
        self.cos, self.sin = tables(table, rotary)
        self.pos = {"index": np.arange(t), "random": rng.integers(0, table, t), "padded": rng.integers(-table, table, t),
                    "padding": np.full(t, -1)}[pos]
        self.pos_d = None if pos == "index" else torch.from_numpy(self.pos.astype(np.int32 if pos == "padded" else np.int64)).cuda()
        self.cos_d, self.sin_d = torch.from_numpy(self.cos).cuda(), torch.from_numpy(self.sin).cuda()

    def tables(self):
        return self.cos_d, self.sin_d, self.pos_d

    def parts(self):
        for x, w, dy in ((self.q, self.wq, self.dq), (self.k, self.wk, self.dk)):
            d = x.shape[-1]
            yield x.float().cpu().numpy(), np.ones(d) if w is None else w.float().cpu().numpy(), dy.float().cpu().numpy()

    def check_forward(self, got):
        for y, (x, w, _) in zip(got, self.parts()):
            close(y, *reference(x, w, self.cos, self.sin, self.pos, self.r, self.interleaved), self.dtype)

    def check_backward(self, got):
        for i, (x, w, dy) in enumerate(self.parts()):
            (dx, bx), (dw, bw) = reference(x, w, self.cos, self.sin, self.pos, self.r, self.interleaved, dy)
            close(got[i], dx, bx, self.dtype)
            if self.wq is None:
                assert got[2 + i] is None
            else:
                assert got[2 + i].dtype == torch.float32
                close(got[2 + i], dw, bw, "f32")

    def forward(self, **kw):
        return hq.hq_qk_norm_rope(self.q, self.k, self.wq, self.wk, *self.tables(), interleaved=self.interleaved, **kw)

    def backward(self, **kw):
        return hq.hq_qk_norm_rope_backward(self.dq, self.dk, self.q, self.k, self.wq, self.wk, *self.tables(),
                                           interleaved=self.interleaved, **kw)


CASES = [
    dict(t=1, heads=1, kv_heads=1, d=2, rotary=2), dict(t=1, heads=32, kv_heads=8, d=128, rotary=128, pos="random"),
    dict(t=3, heads=2, kv_heads=1, d=8, rotary=8), dict(t=5, heads=3, kv_heads=3, d=10, rotary=6, pos="padded"),
    dict(t=33, heads=4, kv_heads=2, d=16, rotary=16), dict(t=9, heads=5, kv_heads=1, d=32, rotary=16, pos="random"),
    dict(t=70, heads=8, kv_heads=8, d=64, rotary=64, pos="padded"), dict(t=50, heads=16, kv_heads=16, d=72, rotary=72, pos="padded"),
    dict(t=21, heads=6, kv_heads=2, d=80, rotary=40), dict(t=40, heads=12, kv_heads=4, d=96, rotary=64, pos="padded"),
    dict(t=64, heads=9, kv_heads=3, d=128, rotary=0, pos="random"), dict(t=19, heads=7, kv_heads=1, d=160, rotary=160),
    dict(t=11, heads=2, kv_heads=2, d=256, rotary=128, pos="random"), dict(t=6, heads=2, kv_heads=1, d=512, rotary=512, pos="random"),
    dict(t=4, heads=1, kv_heads=2, d=514, rotary=258, pos="random"), dict(t=4, heads=2, kv_heads=1, d=1024, rotary=1024, pos="padded"),
    dict(t=7, heads=3, kv_heads=1, d=130, rotary=66, pos="random"), dict(t=700, heads=32, kv_heads=8, d=128, rotary=128, pos="random"),
    dict(t=4, heads=4, kv_heads=1, d=64, rotary=64, pos="padding"), dict(t=1500, heads=3, kv_heads=1, d=40, rotary=20, pos="padded"),
]
# every number of pairs to a lane with every number of lanes to a head, and heads beyond them
CUTS = [dict(t=37, heads=3, kv_heads=1, d=2 * c * (g - g // 4), rotary=2 * c * max(1, g // 2 - 1), pos="padded")
        for c in (1, 2, 4, 8) for g in (2, 4, 8, 16, 32, 64)]
CUTS += [dict(t=13, heads=2, kv_heads=1, d=d, rotary=r, pos="padded") for d, r in
         ((4, 4), (72, 36), (72, 18), (128, 66), (130, 66), (256, 68), (260, 260), (512, 24), (516, 12), (1008, 16), (1024, 8))]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "t%(t)d_h%(heads)d_%(kv_heads)d_d%(d)d_r%(rotary)d" % c)
def test_forward_and_gradients(case, dtype, interleaved):
    c = Case(dtype=dtype, interleaved=interleaved, **case)
    c.check_forward(c.forward())
    got = c.backward()
    c.check_backward(got)
    assert all(torch.equal(a, b) for a, b in zip(got, c.backward()))   # a fixed order: the same bits again


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CUTS, ids=lambda c: "d%(d)d_r%(rotary)d" % c)
def test_cuts_of_a_head(case, dtype, interleaved):
    c = Case(dtype=dtype, interleaved=interleaved, **case)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("weights", ["f32", "none"])
@pytest.mark.parametrize("d,rotary", [(64, 64), (72, 36), (10, 4)])
def test_weights(weights, d, rotary):
    c = Case(20, 4, 2, d, rotary, "bf16", weights=weights, pos="random")
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("d,rotary", [(128, 128), (72, 72), (10, 10)])
def test_in_place_and_strided_results(d, rotary):
    c = Case(130, 6, 2, d, rotary, "f16", pos="padded")
    want, grads = c.forward(), c.backward()
    # into another projection-shaped buffer, heads before tokens, and in place
    buffer = torch.full((130, 10 * d + 3), 9.0, dtype=torch.float16, device="cuda")
    out = (buffer[:, 1:1 + 6 * d].view(130, 6, d), buffer[:, 1 + 6 * d:1 + 8 * d].view(130, 2, d))
    c.forward(out=out)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    assert (buffer[:, 0] == 9).all() and (buffer[:, 1 + 8 * d:] == 9).all()
    turned_out = tuple(torch.empty((h, 130, d), dtype=torch.float16, device="cuda").transpose(0, 1) for h in (6, 2))
    got = c.backward(out=turned_out)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    c.backward(out=(c.dq, c.dk))
    assert torch.equal(c.dq, grads[0]) and torch.equal(c.dk, grads[1])
    c.forward(out=(c.q, c.k))
    assert torch.equal(c.q, want[0]) and torch.equal(c.k, want[1])


def test_repeated_heads_and_gradients():
    """Inputs that share memory: one head seen as several, one gradient for every token."""
    c = Case(20, 4, 2, 64, 64, "f32", pos="random")
    c.q, c.dk = c.q[:, :1].expand(20, 4, 64), c.dk[:1, :1].expand(20, 2, 64)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("d", [64, 10])
def test_positions_beyond_the_tables(d):
    c = Case(6, 2, 1, d, d, "f32", pos="random")
    want = c.forward()
    c.pos_d[2] = c.cos_d.shape[0]
    c.pos_d[4] = 2 ** 62
    got = c.forward()
    for a, b in zip(got, want):
        assert torch.isnan(a[[2, 4]]).all() and torch.equal(a[[0, 1, 3, 5]], b[[0, 1, 3, 5]])


def test_padding_may_hold_anything():
    """Values that are not finite in padding tokens reach neither results nor sums."""
    c = Case(30, 4, 2, 64, 64, "f32", pos="padded")
    want, grads = c.forward(), c.backward()
    pad = torch.from_numpy(c.pos < 0).cuda()
    c.q[pad], c.k[pad] = float("nan"), float("inf")
    c.dq[pad], c.dk[pad] = float("inf"), float("nan")
    assert all(torch.equal(a, b) for a, b in zip(c.forward(), want))
    assert all(torch.equal(a, b) for a, b in zip(c.backward(), grads))


def test_zero_rows_and_scales():
    """A head of zeros; heads of large and of tiny values."""
    c = Case(8, 2, 2, 64, 64, "f32", pos="random")
    c.q[1], c.k[2] = 0, 0
    c.q[3] *= 1e15
    c.k[4] *= 1e-15
    c.check_forward(c.forward())
    c.check_backward(c.backward())


def test_gradients_by_differences():
    c = Case(5, 3, 1, 24, 16, "f32", pos="random", interleaved=True)
    dq, dk, dwq, dwk = (t.cpu().double().numpy() for t in c.backward())
    parts = list(c.parts())

    def loss(i, x, w):
        return (reference(x, w, c.cos, c.sin, c.pos, c.r, True)[0] * parts[i][2]).sum()

    rng = np.random.default_rng(1)
    for i, (dx, dw) in enumerate(((dq, dwq), (dk, dwk))):
        x, w = parts[i][0].astype(np.float64), parts[i][1].astype(np.float64)
        for _ in range(10):
            v, u = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
            h = 1e-5
            # the gradients are fp32 (2^-24 of about 100 terms of size 1), the differences of order h^2 off
            assert abs((loss(i, x + h * v, w) - loss(i, x - h * v, w)) / (2 * h) - (dx * v).sum()) < 1e-4 * np.abs(dx * v).sum()
            assert abs((loss(i, x, w + h * u) - loss(i, x, w - h * u)) / (2 * h) - (dw * u).sum()) < 1e-4 * np.abs(dw * u).sum()


def test_no_tokens():
    c = Case(1, 2, 1, 64, 64, "f16", pos="random")
    c.q, c.k, c.dq, c.dk, c.pos_d = c.q[:0], c.k[:0], c.dq[:0], c.dk[:0], c.pos_d[:0]
    q, k = c.forward()
    assert q.shape == (0, 2, 64) and k.shape == (0, 1, 64)
    dq, dk, dwq, dwk = c.backward()
    assert dq.shape == (0, 2, 64) and not dwq.any() and not dwk.any()


def test_another_stream_and_a_graph():
    c = Case(300, 8, 2, 128, 128, "bf16", pos="random")
    step = lambda: c.forward() + c.backward()
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        c.q.mul_(0.5)
        want = [t.clone() for t in step()]


def test_refusals():
    c = Case(6, 4, 2, 64, 64, "f16", pos="random")
    call = lambda **kw: hq.hq_qk_norm_rope(*[kw.get(n, d) for n, d in (
        ("q", c.q), ("k", c.k), ("wq", c.wq), ("wk", c.wk), ("cos", c.cos_d), ("sin", c.sin_d), ("pos", c.pos_d))], **kw.get("more", {}))
    call()
    bad = [dict(q=c.q.cpu()), dict(q=c.q[0]), dict(q=c.q.double()), dict(k=c.k.float()), dict(k=c.k[:5]), dict(k=c.k[..., :32]),
           dict(q=c.q.transpose(1, 2)), dict(q=c.q[..., ::2], k=c.k[..., ::2]), dict(wq=c.wq[:32]), dict(wq=c.wq.double()),
           dict(wq=c.wq.float()), dict(cos=c.cos_d.half()), dict(cos=c.cos_d[:3]), dict(cos=c.cos_d[0], sin=c.sin_d[0]),
           dict(pos=c.pos_d[:5]), dict(pos=c.pos_d.float()), dict(more=dict(out=(c.q, c.q))),
           dict(more=dict(out=(c.q[:1].expand(6, 4, 64), c.k)))]
    for i, kw in enumerate(bad):
        with pytest.raises(ValueError):
            call(**kw)
            pytest.fail("case %d was not refused" % i)
    wide, wide_s = (t.repeat(1, 2) for t in (c.cos_d, c.sin_d))
    for kw, code in ((dict(cos=wide, sin=wide_s), 2),                                   # more rotated channels than there are
                     (dict(pos=None, cos=c.cos_d[:5], sin=c.sin_d[:5]), 2),             # tables shorter than the sequence
                     (dict(more=dict(eps=-1.0)), 2), (dict(more=dict(eps=float("nan"))), 2),
                     (dict(q=c.q[..., :63], k=c.k[..., :63], wq=None, wk=None), 2)):    # an odd head
        with pytest.raises(hq.HqError) as e:
            call(**kw)
        assert e.value.code == code
    with pytest.raises(ValueError):
        hq.hq_qk_norm_rope_backward(c.dq[:, :3], c.dk, c.q, c.k, c.wq, c.wk, *c.tables())


def test_results_that_share_memory():
    """Results that lie on each other or on another input than their own are refused; views of one buffer that lie between each other are not."""
    t, h, d = 50, 4, 64
    c = Case(t, h, h, d, d, "f16", pos="random")
    free = lambda: torch.empty((t, h, d), dtype=torch.float16, device="cuda")
    flat = torch.zeros(t * h * d + 32, dtype=torch.float16, device="cuda")
    table_f16 = c.cos_d.view(torch.float16).flatten()
    one = c.cos_d.shape[0] * d // (h * d)   # tokens whose results would fit the table
    bad = [(c.q, c.q), (c.k, c.q), (c.k, free()), (free(), c.q), (flat[:t * h * d].view(t, h, d), flat[32:].view(t, h, d)), (c.k, c.k),
           (flat[:t * h * d].view(t, h, d), flat[:t * h * d].view(h, t, d).transpose(0, 1))]
    keep = c.q.clone(), c.k.clone(), flat.clone()
    for i, out in enumerate(bad):
        with pytest.raises(ValueError, match="must not overlap"):
            c.forward(out=out)
            pytest.fail("case %d was not refused" % i)
    for i, out in enumerate(bad + [(c.dk, c.dq), (c.dk, free()), (free(), c.dq), (c.dq, c.q)]):
        with pytest.raises(ValueError, match="must not overlap"):
            c.backward(out=out)
            pytest.fail("case %d was not refused" % i)
    # q moved on by a head, and onto the tables and the weights
    wide = torch.zeros((t, (h + 1) * d), dtype=torch.float16, device="cuda")
    for args, out in (((wide[:, :h * d].view(t, h, d), c.k), (wide[:, d:].view(t, h, d), free())),
                      ((c.q[:one], c.k[:one]), (table_f16[:one * h * d].view(one, h, d), free()[:one])),
                      ((c.q[:1, :1], c.k[:1, :1]), (free()[:1, :1], c.wk.view(1, 1, d)))):
        n = args[0].shape[0]
        with pytest.raises(ValueError, match="must not overlap"):
            hq.hq_qk_norm_rope(*args, c.wq, c.wk, c.cos_d, c.sin_d, c.pos_d[:n], out=out)
    assert all(torch.equal(a, b) for a, b in zip((c.q, c.k, flat), keep))

    # accepted: in place in one projection's result, whose heads or parts follow one another; results between other results' rows
    want, grads = c.forward(), c.backward()
    for layout in ((t, 3, h, d), (t, h, 3, d)):
        part = lambda b, i: b.select(layout.index(3), i)
        qkv, dqkv = (torch.zeros(layout, dtype=torch.float16, device="cuda") for _ in range(2))
        for b, x, y in ((qkv, c.q, c.k), (dqkv, c.dq, c.dk)):
            part(b, 0).copy_(x)
            part(b, 1).copy_(y)
        args = (part(qkv, 0), part(qkv, 1), c.wq, c.wk, *c.tables())
        got = hq.hq_qk_norm_rope_backward(part(dqkv, 0), part(dqkv, 1), *args, out=(part(dqkv, 0), part(dqkv, 1)))
        assert torch.equal(part(dqkv, 0), grads[0]) and torch.equal(part(dqkv, 1), grads[1]) and torch.equal(got[2], grads[2])
        assert not part(dqkv, 2).any()
        hq.hq_qk_norm_rope_backward(c.dq, c.dk, *args, out=(part(dqkv, 2), part(dqkv, 1)))
        assert torch.equal(part(dqkv, 2), grads[0])
        hq.hq_qk_norm_rope(*args, out=args[:2])
        assert torch.equal(part(qkv, 0), want[0]) and torch.equal(part(qkv, 1), want[1]) and not part(qkv, 2).any()
    both = torch.empty((2 * h, t, d), dtype=torch.float16, device="cuda")
    out = both[0::2].transpose(0, 1), both[1::2].transpose(0, 1)
    c.forward(out=out)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    c.backward(out=(c.q, c.dk))
    assert torch.equal(c.q, grads[0]) and torch.equal(c.dk, grads[1])


def test_refusals_of_gradients():
    c = Case(6, 4, 2, 64, 64, "f16", pos="random")
    odd = [x[..., :63] for x in (c.dq, c.dk, c.q, c.k)]
    wide = [torch.zeros((6, h, 1026), dtype=torch.float16, device="cuda") for h in (4, 2, 4, 2)]
    whole = [c.dq, c.dk, c.q, c.k]
    for tensors, tables, more, code in ((odd, c.tables(), {}, 2), (wide, c.tables(), {}, 6), (whole, [t.repeat(1, 2) for t in c.tables()[:2]], {}, 2),
                                        (whole, [t[:5] for t in c.tables()[:2]], {}, 2), (whole, c.tables(), dict(eps=-1.0), 2)):
        with pytest.raises(hq.HqError) as e:
            hq.hq_qk_norm_rope_backward(*tensors, None, None, *tables, **more)
        assert e.value.code == code
