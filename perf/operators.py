"""Cases that time the operators of transformer blocks: layers of 8-bit floats with block scales, and the norm and
rotation of queries and keys.

A case is one pass through one operator on data that a program has in hand:

op           one pass
linear       y = x W^T + bias: the activations are quantised to E4M3 with one scale for each token and 128 channels, the
             weights are held as E4M3 codes with one scale for each block of 128 x 128
linear_grad  the gradients of that layer: dx from dy (quantised along the outputs) and the weights' codes, dW from dy and x
             (both quantised along the tokens, dy with one scale for each output and 128 tokens, x with one for each block of
             128 x 128), dbias
qk           q and k, views of one projection's result, each head normalised (root mean square, a weight for each channel)
             and rotated by its token's position
qk_grad      the gradients of that with respect to q, k and the two weights

`own` chooses between elementary torch operations in 32 bits (false) and the framework's calls (true).
"""
import math

import numpy as np
import torch

own = False

GROUP = 128           # elements that share a scale
E4M3_MAX = 448.0
EPS = 1e-6
_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def _linear(m, k, n, dtype, bias=False, op="linear"):
    return {"op": op, "m": m, "k": k, "n": n, "dtype": dtype, "bias": bias}


def _qk(t, heads, kv_heads, d, rotary, dtype, sequences=1, interleaved=False, padding=False, op="qk"):
    return {"op": op, "t": t, "heads": heads, "kv_heads": kv_heads, "d": d, "rotary": rotary, "dtype": dtype,
            "sequences": sequences, "interleaved": interleaved, "padding": padding}


def listed():
    cases = [
        # one row through the widest feed-forward layer of the benchmark configurations, as a timestep's embedding or a
        # single decoded token takes it: latency counts
        ("linear_one_row", _linear(1, 960, 3840, "bf16", bias=True)),
        # a ragged layer: no size is a multiple of anything, rows of x are not aligned to 16 bytes
        ("linear_ragged", _linear(333, 1001, 777, "f16", bias=True)),
        # the query/key/value projection of an attention block of the benchmark configurations
        ("linear_qkv", _linear(16 * 16 * 16, 576, 1728, "f16")),
        # a large feed-forward layer over a long batch of tokens
        ("linear_large", _linear(8192, 4096, 8192, "bf16")),
        # gradients of a ragged layer with fp32 activations
        ("linear_grad_ragged", _linear(300, 520, 264, "f32", bias=True, op="linear_grad")),
        # gradients of the widest feed-forward layer of the benchmark configurations
        ("linear_grad_ffn", _linear(2048, 960, 3840, "f16", bias=True, op="linear_grad")),
        # gradients of a large projection over a long batch of tokens
        ("linear_grad_large", _linear(8192, 4096, 4096, "bf16", op="linear_grad")),
        # one decoded token, grouped key heads
        ("qk_one_token", _qk(1, 32, 8, 128, 128, "bf16")),
        # image tokens of a diffusion transformer, 72 channels a head, several images with padding between them
        ("qk_ragged", _qk(1021, 16, 16, 72, 72, "f16", sequences=5, padding=True)),
        # a long prompt with grouped key heads
        ("qk_large", _qk(65536, 32, 8, 128, 128, "bf16", sequences=8)),
        # training on a ragged batch, partly rotated heads, neighbouring channels paired
        ("qk_grad_ragged", _qk(1333, 12, 4, 96, 64, "f32", sequences=3, interleaved=True, padding=True, op="qk_grad")),
        # training on a long batch
        ("qk_grad_large", _qk(32768, 32, 8, 128, 128, "bf16", sequences=16, op="qk_grad")),
    ]
    return [dict(c, name=name) for name, c in cases]


def _spread(rng, low, high):
    """A whole number, uniform in the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["linear", "linear_grad", "qk", "qk_grad"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    if op == "linear":
        return _linear(_spread(rng, 1, 8192), _spread(rng, 64, 4096), _spread(rng, 64, 8192), dtype, rng.random() < 0.5)
    if op == "linear_grad":
        return _linear(_spread(rng, 32, 8192), _spread(rng, 64, 4096), _spread(rng, 64, 4096), dtype, rng.random() < 0.5,
                       op=op)
    d = rng.choice([32, 40, 64, 72, 80, 96, 128, 160, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv_heads * rng.choice([1, 2, 4])
    rotary = rng.choice([d, d, d // 2])
    # as many elements at most as the largest listed case has
    most = (65536 if op == "qk" else 32768) * 40 * 128 * 2 // (_SIZE[dtype] * (heads + kv_heads) * d)
    t = _spread(rng, 1, min(65536 if op == "qk" else 32768, most))
    return _qk(t, heads, kv_heads, d, rotary, dtype, rng.randint(1, min(t, 16)), rng.random() < 0.3, rng.random() < 0.3, op)


# ---- what a program has in hand ---------------------------------------------------------------------------------

def _values(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale


def _activations(gen, m, k):
    """Normal values; one channel in a hundred is larger by 20, for every token."""
    x = _values(gen, (m, k))
    channels = torch.randperm(k, generator=gen, device="cuda")[:max(1, k // 100)]
    x[:, channels] *= 20.0
    return x


def _ceil(a, b):
    return -(-a // b)


def _pad(t, rows, columns):
    out = t.new_zeros((rows, columns))
    out[:t.shape[0], :t.shape[1]] = t
    return out


def _scale_of(amax):
    """The scale of values whose largest magnitude is amax: 1 where all are zero, never below the smallest normal number."""
    return torch.where(amax == 0, torch.ones_like(amax), torch.clamp(amax / E4M3_MAX, min=2.0 ** -126))


def _codes(x, scale):
    return (x * (1.0 / scale)).to(torch.float8_e4m3fn)


def _block_codes(w):
    """E4M3 codes [n, k up to a multiple of 16] and scales [n / 128, k / 128] of w [n, k]; the rows' ends hold zeros."""
    n, k = w.shape
    nb, kb = _ceil(n, GROUP), _ceil(k, GROUP)
    blocks = _pad(w.float(), nb * GROUP, kb * GROUP).view(nb, GROUP, kb, GROUP)
    scale = _scale_of(blocks.abs().amax(dim=(1, 3)))
    codes = _codes(blocks, scale[:, None, :, None]).view(torch.uint8).view(nb * GROUP, kb * GROUP)
    return codes[:n, :_ceil(k, 16) * 16].contiguous().view(torch.float8_e4m3fn), scale


def _transposed_codes(codes, n, k):
    """The codes of the transposed weights, rows up to a multiple of 16."""
    out = torch.zeros((k, _ceil(n, 16) * 16), dtype=torch.uint8, device=codes.device)
    out[:, :n] = codes.view(torch.uint8)[:, :k].t()
    return out.view(torch.float8_e4m3fn)


def _positions(case, rng):
    """Positions that restart with each sequence; with padding, the last tokens of each sequence are -1."""
    cuts = np.sort(rng.choice(np.arange(1, case["t"]), case["sequences"] - 1, replace=False)) if case["sequences"] > 1 else []
    ends = np.concatenate([cuts, [case["t"]]]).astype(np.int64)
    begins = np.concatenate([[0], ends[:-1]])
    pos = np.arange(case["t"], dtype=np.int64) - np.repeat(begins, ends - begins)
    if case["sequences"] == 1:
        pos += int(rng.integers(0, 4096))       # a token of a conversation that has gone on for a while
    if case["padding"]:
        length = np.repeat(ends - begins, ends - begins)
        pos = np.where(pos - pos.min() >= np.ceil(length * 0.9), -1, pos)
    return pos


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPE[case["dtype"]]
    s = dict(case)
    if case["op"] in ("linear", "linear_grad"):
        m, k, n = case["m"], case["k"], case["n"]
        s["x"] = _activations(gen, m, k).to(dt)
        s["wq"], s["w_scale"] = _block_codes(_values(gen, (n, k), 0.02))
        s["b"] = _values(gen, (n,), 0.01).to(dt) if case["bias"] else None
        if case["op"] == "linear_grad":
            s["dy"] = _values(gen, (m, n), 1e-3).to(dt)
            s["wq_t"] = _transposed_codes(s.pop("wq"), n, k)
        return s
    t, h, hk, d, r = (case[i] for i in ("t", "heads", "kv_heads", "d", "rotary"))
    pos = _positions(case, np.random.default_rng(seed))
    s["positions"] = torch.from_numpy(pos).cuda()
    angles = torch.outer(torch.arange(int(pos.max()) + 1, dtype=torch.float64),
                         10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r))
    s["cos"], s["sin"] = angles.cos().float().cuda(), angles.sin().float().cuda()
    qkv = (_values(gen, (t, (h + 2 * hk) * d)) * 2.0).to(dt)
    s["q"] = qkv[:, :h * d].view(t, h, d)
    s["k"] = qkv[:, h * d:(h + hk) * d].view(t, hk, d)
    s["q_weight"] = (1.0 + _values(gen, (d,), 0.1)).to(dt)
    s["k_weight"] = (1.0 + _values(gen, (d,), 0.1)).to(dt)
    if case["op"] == "qk_grad":
        s["dq"] = _values(gen, (t, h, d), 1e-2).to(dt)
        s["dk"] = _values(gen, (t, hk, d), 1e-2).to(dt)
    return s


# ---- one pass: the framework's calls ------------------------------------------------------------------------------

def _run_own(s):
    import paper_2512_05746_amd as hq
    if s["op"] == "linear":
        return hq.hq_act_quant_fp8_linear(s["x"], s["wq"], s["w_scale"], s["b"], y_dtype=s["x"].dtype)
    if s["op"] == "linear_grad":
        return hq.hq_fp8_linear_backward(s["dy"], s["x"], s["wq_t"], s["w_scale"], bias_grad=s["bias"])
    if s["op"] == "qk":
        return hq.hq_qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], s["positions"],
                                  eps=EPS, interleaved=s["interleaved"])
    return hq.hq_qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"],
                                       s["positions"], eps=EPS, interleaved=s["interleaved"])


# ---- one pass: elementary operations in 32 bits -------------------------------------------------------------------

def _dequantised_rows(x):
    """x [r, c] after quantisation with one scale for each row and 128 columns."""
    r, c = x.shape
    cb = _ceil(c, GROUP)
    g = _pad(x, r, cb * GROUP).view(r, cb, GROUP)
    scale = _scale_of(g.abs().amax(-1))[..., None]
    return (_codes(g, scale).float() * scale).view(r, cb * GROUP)[:, :c]


def _dequantised_blocks(x):
    """x [r, c] after quantisation with one scale for each block of 128 x 128."""
    r, c = x.shape
    rb, cb = _ceil(r, GROUP), _ceil(c, GROUP)
    g = _pad(x, rb * GROUP, cb * GROUP).view(rb, GROUP, cb, GROUP)
    scale = _scale_of(g.abs().amax(dim=(1, 3)))[:, None, :, None]
    return (_codes(g, scale).float() * scale).view(rb * GROUP, cb * GROUP)[:r, :c]


def _weights(codes, scale, n, k):
    """The values that codes [n, ..] stand for; scale [n / 128, k / 128]."""
    each = scale.repeat_interleave(GROUP, 0)[:n].repeat_interleave(GROUP, 1)[:, :k]
    return codes.float()[:, :k] * each


def _rotated(n, cos, sin, r, interleaved):
    """n [t, h, d], its first r channels rotated by cos, sin [t, 1, r / 2]."""
    a, b = (n[..., 0:r:2], n[..., 1:r:2]) if interleaved else (n[..., :r // 2], n[..., r // 2:r])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, n[..., r:]], -1)


def _run_plain(s):
    if s["op"] == "linear":
        w = _weights(s["wq"], s["w_scale"], s["n"], s["k"])
        y = torch.mm(_dequantised_rows(s["x"].float()), w.t())
        return (y if s["b"] is None else y + s["b"].float()).to(s["x"].dtype)
    if s["op"] == "linear_grad":
        x, dy = s["x"].float(), s["dy"].float()
        wt = _weights(s["wq_t"], s["w_scale"].t(), s["k"], s["n"])
        dx = torch.mm(_dequantised_rows(dy), wt.t()).to(s["x"].dtype)
        dw = torch.mm(_dequantised_rows(dy.t()), _dequantised_blocks(x))
        return dx, dw, dy.sum(0) if s["bias"] else None
    live = (s["positions"] >= 0)[:, None, None]
    at = s["positions"].clamp(min=0)
    cos, sin, r = s["cos"][at][:, None, :], s["sin"][at][:, None, :], s["rotary"]
    out, sums = [], []
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"].float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if s["op"] == "qk":
            y = _rotated(x * rstd * w, cos, sin, r, s["interleaved"])
            out.append(torch.where(live, y, 0.0).to(s[name].dtype))
            continue
        g = torch.where(live, _rotated(s["d" + name].float(), cos, -sin, r, s["interleaved"]), 0.0)
        unit = x * rstd
        sums.append((g * unit).sum((0, 1)))
        g = g * w
        dx = rstd * (g - unit * (g * unit).mean(-1, keepdim=True))
        out.append(dx.to(s[name].dtype))
    return tuple(out + sums)


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _e4m3(v):
    """v rounded to the nearest E4M3 number (3 bits of mantissa, exponents from -6, subnormals below), ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantised(x, rows):
    """Values after quantisation in tiles of rows x 128, in 64 bits."""
    r, c = x.shape
    tile = torch.nn.functional.pad(x, (0, -c % GROUP, 0, -r % rows))
    shape = tile.shape
    tile = tile.reshape(shape[0] // rows, rows, shape[1] // GROUP, GROUP)
    top = tile.abs().amax((1, 3), keepdim=True)
    s = torch.where(top > 0, top / E4M3_MAX, 1.0)
    return (_e4m3(tile / s) * s).reshape(shape)[:r, :c]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("linear", "linear_grad"):
        m, k, n = case["m"], case["k"], case["n"]
        x = s["x"].double()
        row, column = torch.arange(n, device="cuda") // GROUP, torch.arange(k, device="cuda") // GROUP
        scale = s["w_scale"].double()[row][:, column]
        if case["op"] == "linear":
            w = s["wq"].double()[:, :k] * scale
            y = _exact_quantised(x, 1) @ w.T
            return y + s["b"].double() if s["b"] is not None else y
        w, dy = s["wq_t"].double()[:, :n].T * scale, s["dy"].double()
        dw = _exact_quantised(dy.T.contiguous(), 1) @ _exact_quantised(x, GROUP)
        return _exact_quantised(dy, 1) @ w, dw, torch.ones(m, dtype=torch.float64, device="cuda") @ dy if case["bias"] else None
    r = case["rotary"]
    pos = s["positions"]
    # as complex numbers: channel pair i of a token is multiplied by cos + i sin
    turn = torch.complex(s["cos"].double(), s["sin"].double())[pos.clamp(min=0)][:, None]
    turn = turn * (pos >= 0)[:, None, None]
    keep = (pos >= 0)[:, None, None].double()

    def pairs(v):
        a, b = (v[..., 0:r:2], v[..., 1:r:2]) if case["interleaved"] else (v[..., :r // 2], v[..., r // 2:r])
        return torch.complex(a.contiguous(), b.contiguous())

    def turned(v, by):
        z = pairs(v) * by
        out = v * keep
        if case["interleaved"]:
            out[..., 0:r:2], out[..., 1:r:2] = z.real, z.imag
        else:
            out[..., :r // 2], out[..., r // 2:r] = z.real, z.imag
        return out

    first, second = [], []
    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "_weight"].double()
        norm = (x.square().sum(-1, keepdim=True) / case["d"] + EPS).sqrt()
        if case["op"] == "qk":
            first.append(turned(x / norm * w, turn))
            continue
        g = turned(s["d" + name].double(), turn.conj())
        second.append((g * x / norm).sum((0, 1)))
        g = g * w
        first.append(g / norm - x * (g * x).sum(-1, keepdim=True) / (case["d"] * norm ** 3))
    return tuple(first + second)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] in ("linear", "linear_grad"):
        m, k, n = case["m"], case["k"], case["n"]
        scales = 4 * _ceil(k, GROUP) * _ceil(n, GROUP)
        bias = n * (size if case["op"] == "linear" else 4) if case["bias"] else 0
        if case["op"] == "linear":
            return {"bytes": m * k * size + n * k + scales + bias + m * n * size, "flops": 2 * m * n * k}
        # x and dy read, the codes read, dx and dW written
        return {"bytes": 2 * m * k * size + m * n * size + n * k + scales + 4 * n * k + bias, "flops": 4 * m * n * k}
    rows = case["t"] * (case["heads"] + case["kv_heads"])
    elements = rows * case["d"]
    tables = 4 * case["rotary"] * -(-case["t"] // case["sequences"]) + 8 * case["t"]
    weights = 2 * case["d"] * size
    if case["op"] == "qk":
        return {"bytes": 2 * elements * size + tables + weights, "flops": 8 * elements}
    return {"bytes": 3 * elements * size + tables + weights + 8 * case["d"], "flops": 16 * elements}
