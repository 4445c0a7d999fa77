"""Cases that time the operators of a key/value cache held in 4 bits: appending to it, attention over it, reading it back.

The cache is paged.  A head of a token is H y (H the orthonormal block-diagonal Hadamard matrix, symmetric and its own inverse), as
E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one fp32 scale:

k        [pages, kv_heads, page_size, pitch / 2] bytes; channel 2 i of a token in the low bits of byte i
v        [pages, kv_heads, page_size / 8, pitch, 4] bytes: a channel's codes of 8 tokens side by side, the first in the low bits
k_scale, v_scale   [pages, kv_heads, page_size] fp32

Sequence b has lengths[b] tokens in the cache, the newest of them the tokens of the call; page_table[b] names its pages.

op        one pass
append    query and key heads are normalised (where the case has a norm) and rotated by their positions; keys and values go into the
          cache.  Gives the queries, and the keys and values that the cache now holds for these tokens, read back in 16 bits
read      the keys and values of all cached tokens
attend    each query head over the tokens of its sequence up to its own position, or over the last `window` of them and the
          first `sinks`

`own` chooses between elementary torch operations (false: products in 32 bits, what decides a code in 64) and the framework's calls
(true).
"""
import math

import torch

own = False

EPS = 1e-6
E2M1_MAX = 6.0
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def _case(op, batch, tokens, cached, heads, kv_heads, d, dtype, page=64, ragged=False, rotary=0, norm=True, interleaved=False,
          window=0, sinks=0, padding=0):
    return {"op": op, "batch": batch, "tokens": tokens, "cached": cached, "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype,
            "page": page, "ragged": ragged, "rotary": rotary, "norm": norm, "interleaved": interleaved, "window": window,
            "sinks": sinks, "padding": padding}


def listed():
    cases = [
        # one new token for each of a few conversations: latency counts
        ("append_step", _case("append", 16, 1, 4096, 32, 8, 128, "bf16", rotary=128)),
        # chunks of several lengths in one padded batch, few channels rotated, neighbours paired, no norm, small pages
        ("append_ragged", _case("append", 5, 300, 900, 12, 4, 80, "f32", page=16, ragged=True, rotary=40, norm=False, interleaved=True,
                                padding=7)),
        # long prompts
        ("append_prompt", _case("append", 4, 8192, 0, 32, 8, 128, "bf16", rotary=128)),
        # a few short sequences taken out of the cache
        ("read_ragged", _case("read", 7, 0, 1200, 16, 16, 80, "f16", page=16, ragged=True)),
        # a long document taken out of the cache
        ("read_long", _case("read", 1, 0, 131072, 32, 8, 128, "bf16")),
        # one token of one conversation: latency counts
        ("attend_one_token", _case("attend", 1, 1, 776, 32, 8, 128, "bf16", page=16)),
        # a batch of conversations of all lengths, a token each
        ("attend_batch", _case("attend", 64, 1, 16384, 32, 8, 128, "bf16", ragged=True)),
        # a token over a very long document
        ("attend_long", _case("attend", 1, 1, 262143, 32, 8, 128, "bf16")),
        # long conversations of which the last thousand tokens and the first four stay visible
        ("attend_window", _case("attend", 48, 1, 32768, 64, 8, 64, "f16", ragged=True, window=1024, sinks=4)),
        # a few drafted tokens checked at once, in 32 bits
        ("attend_drafts", _case("attend", 12, 5, 3001, 24, 8, 96, "f32", page=32, ragged=True)),
        # chunks and single tokens in one padded batch, every head with keys of its own
        ("attend_mixed", _case("attend", 12, 700, 2500, 16, 16, 80, "f16", page=16, ragged=True, padding=13)),
        # the second half of long prompts
        ("attend_prompt", _case("attend", 2, 4096, 4096, 32, 8, 128, "bf16")),
    ]
    return [dict(c, name=name) for name, c in cases]


def _spread(rng, low, high):
    """A whole number, uniform in the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    d = rng.choice([32, 48, 64, 80, 96, 112, 128, 160, 192, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    ragged = rng.random() < 0.6
    padding = rng.choice([0, 0, 1, 9])
    if op == "append":
        batch = _spread(rng, 1, 64)
        rows = 32768 * 48 * 128 // ((heads + 2 * kv_heads) * d * _SIZE[dtype] // 2)
        tokens = 1 if rng.random() < 0.3 else _spread(rng, 1, max(1, min(8192, rows // batch)))
        return _case(op, batch, tokens, rng.choice([0, _spread(rng, 1, 4096)]), heads, kv_heads, d, dtype, page, ragged and tokens > 1,
                     rng.choice([0, d // 2, d, d]), rng.random() < 0.7, rng.random() < 0.3, padding=padding if tokens > 1 else 0)
    if op == "read":
        batch = _spread(rng, 1, 32)
        most = 131072 * 8 * 128 // (kv_heads * d * batch * _SIZE[dtype] // 2)
        return _case(op, batch, 0, _spread(rng, 1, max(1, min(65536, most))), heads, kv_heads, d, dtype, page, ragged)
    window, sinks = rng.choice([(0, 0), (0, 0), (_spread(rng, 1, 4096), rng.choice([0, 4, 17]))])
    batch = _spread(rng, 1, 64)
    if rng.random() < 0.5:              # a token or a few drafted ones for each sequence
        tokens = rng.choice([1, 1, 1, 2, 3, 7])
        most = 262144 * 8 * 128 // (kv_heads * d * batch)
        return _case(op, batch, tokens, _spread(rng, 1, max(1, min(262144, most))), heads, kv_heads, d, dtype, page, ragged,
                     window=window, sinks=sinks)
    batch = min(batch, 12)
    tokens = _spread(rng, 8, 4096)
    cached = rng.choice([0, _spread(rng, 1, 4096)])
    # (query head, token) pairs, 32-bit types at a third
    pairs = 2 * 32 * 4096 * 6144 * 128 // d // (3 if dtype == "f32" else 1)
    while batch * heads * tokens * (tokens + cached) > pairs:
        tokens, cached = max(1, tokens // 2), cached // 2
    return _case(op, batch, tokens, cached, heads, kv_heads, d, dtype, page, ragged, window=window, sinks=sinks, padding=padding)


# ---- what a program has in hand ---------------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _block(d):
    """The largest power of two that divides d, 128 at most: a block of the Hadamard matrix."""
    return min(128, d & -d)


def _sequences(case):
    """(new tokens, tokens in the cache with them) of each sequence.  Ragged: spread evenly over the logarithm, in mixed order."""
    def each(most, least, turn):
        if not case["ragged"] or case["batch"] == 1 or most <= least:
            return [most] * case["batch"]
        at = [(i * 7 + turn) % case["batch"] if case["batch"] % 7 else (i * 5 + turn) % case["batch"] for i in range(case["batch"])]
        low = max(least, most // 64, 1)
        return [int(round(low * (most / low) ** (i / (case["batch"] - 1)))) for i in at]

    new, old = each(case["tokens"], 1, 0), each(case["cached"], 0, case["batch"] // 2)
    return new, [n + c for n, c in zip(new, old)]


def _total(case):
    """Tokens of a call."""
    new, lengths = _sequences(case)
    return sum(lengths) if case["op"] == "read" else sum(new) + case["padding"]


def _hadamard(d, dtype):
    """[d, d], symmetric, its own inverse."""
    h = torch.ones((1, 1), dtype=dtype, device="cuda")
    while h.shape[0] < _block(d):
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0) * math.sqrt(0.5)
    return torch.block_diag(*[h] * (d // _block(d)))


def _codes(z):
    """E2M1 codes and scales of heads z [.., d], to nearest, ties to even."""
    amax = z.abs().amax(-1, keepdim=True)
    scale = torch.where(amax == 0, torch.ones_like(amax), torch.clamp(amax / E2M1_MAX, min=2.0 ** -126)).float()
    t = z * (1.0 / scale)
    a = t.abs()
    code = (t < 0).to(torch.uint8) * 8
    for border in (0.25, 1.25, 2.5, 5.0):       # the number below is even
        code += a > border
    for border in (0.75, 1.75, 3.5):
        code += a >= border
    return code, scale[..., 0]


def _cache(case, seed, pages):
    """A cache whose pages hold normal values."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    hk, d, ps = case["kv_heads"], case["d"], case["page"]
    pitch = _ceil(d, 32) * 32
    k = torch.zeros((pages, hk, ps, pitch // 2), dtype=torch.uint8, device="cuda")
    v = torch.zeros((pages, hk, ps // 8, pitch, 4), dtype=torch.uint8, device="cuda")
    k_scale = torch.zeros((pages, hk, ps), device="cuda")
    v_scale = torch.zeros((pages, hk, ps), device="cuda")
    step = max(1, (1 << 25) // (hk * ps * d))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        code, k_scale[p:p + n] = _codes(torch.randn((n, hk, ps, d), generator=gen, device="cuda"))
        k[p:p + n, :, :, :d // 2] = code[..., 0::2] | code[..., 1::2] << 4
        code, v_scale[p:p + n] = _codes(torch.randn((n, hk, ps, d), generator=gen, device="cuda"))
        code = code.view(n, hk, ps // 8, 8, d).transpose(3, 4)
        v[p:p + n, :, :, :d] = code[..., 0::2] | code[..., 1::2] << 4
    return {"k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    dt, h, hk, d, ps = _DTYPE[case["dtype"]], case["heads"], case["kv_heads"], case["d"], case["page"]
    new, lengths = _sequences(case)
    need = [_ceil(n, ps) for n in lengths]
    order = torch.randperm(sum(need) + 3, generator=gen, device="cuda").int()
    table = torch.full((case["batch"], max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["cache"] = _cache(case, seed, sum(need) + 3)
    s["page_table"], s["lengths"] = table, torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["t"] = t = _total(case)
    s["most_new"], s["longest"] = max(new), max(lengths)
    each = lengths if case["op"] == "read" else new
    s["begins"] = None
    if case["ragged"] or case["padding"]:
        s["begins"] = torch.tensor([0] + each, dtype=torch.int32, device="cuda").cumsum(0).int()
    if case["op"] == "read":
        s["most_new"] = max(lengths)
    elif case["op"] == "append":
        qkv = (torch.randn((t, (h + 2 * hk) * d), generator=gen, device="cuda") * 2.0).to(dt)
        s["q"] = qkv[:, :h * d].view(t, h, d)
        s["k"] = qkv[:, h * d:(h + hk) * d].view(t, hk, d)
        s["v"] = qkv[:, (h + hk) * d:].view(t, hk, d)
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"] = (1.0 + 0.1 * torch.randn((d,), generator=gen, device="cuda")).to(dt)
            s["k_weight"] = (1.0 + 0.1 * torch.randn((d,), generator=gen, device="cuda")).to(dt)
        r = case["rotary"]
        angles = torch.outer(torch.arange(max(lengths), dtype=torch.float64),
                             10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / max(r, 1)))
        s["cos"], s["sin"] = angles.cos().float().cuda(), angles.sin().float().cuda()
    else:
        s["q"] = (torch.randn((t, h, d), generator=gen, device="cuda") * 2.0).to(dt)
    return s


# ---- one pass: the framework's calls ------------------------------------------------------------------------------

def _run_own(s):
    import paper_2512_05746_amd as hq
    c = s["cache"]
    cache = hq.Kv4Cache(c["k"], c["v"], c["k_scale"], c["v_scale"], s["d"])
    if s["op"] == "attend":
        return hq.hq_kv4_attention(s["q"], cache, s["page_table"], s["lengths"], s["begins"], window=s["window"], sinks=s["sinks"])
    if s["op"] == "read":
        return hq.hq_kv4_read(cache, s["page_table"], s["lengths"], s["t"], s["begins"], y_dtype=_DTYPE[s["dtype"]])
    q = hq.hq_kv4_append(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], cache, s["page_table"], s["lengths"],
                         s["begins"], eps=EPS if s["norm"] else None, interleaved=s["interleaved"])
    return (q,) + hq.hq_kv4_read(cache, s["page_table"], s["lengths"], s["t"], s["begins"], y_dtype=_stored(s))


def _stored(s):
    """The type in which what an append stored is looked at."""
    return _DTYPE["bf16" if s["dtype"] == "f32" else s["dtype"]]


# ---- one pass: elementary operations ------------------------------------------------------------------------------

def _places(s, each):
    """For tokens 0 .. t - 1, `each` of them (a number, or what s["begins"] says) to a sequence: the sequence (0 for those of none),
    whether there is one, and the place inside the sequence's new tokens, counted from the end of the sequence."""
    at = torch.arange(s["t"], device="cuda")
    if s["begins"] is None:
        b = at // each
        return b, torch.ones_like(at, dtype=torch.bool), (b + 1) * each - at
    b = torch.searchsorted(s["begins"][1:].contiguous(), at.int(), right=True)
    live = b < s["batch"]
    b = torch.where(live, b, 0)
    return b, live, s["begins"].long()[b + 1] - at


def _nibbles(x):
    """Bytes [.., n] as codes [.., 2 n]."""
    return torch.stack([x & 15, x >> 4], -1).flatten(-2)


def _numbers(codes):
    values = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device="cuda")
    return values[codes.int()]


def _read_plain(s, dtype):
    """(k, v) [t, kv_heads, d] of the tokens of the call."""
    c, ps, d = s["cache"], s["page"], s["d"]
    b, live, back = _places(s, s["most_new"])
    pos = torch.where(live, s["lengths"][b].long() - back, 0)
    page, slot = s["page_table"][b, pos // ps].long(), pos % ps
    hd = _hadamard(d, torch.float32)
    live = live[:, None, None]
    k = _numbers(_nibbles(c["k"][page, :, slot]))[..., :d] * c["k_scale"][page, :, slot][..., None]
    byte = c["v"].transpose(3, 4)[page, :, slot // 8, (slot % 8) // 2]                       # [t, kv_heads, pitch]
    v = _numbers(byte >> (slot % 2 * 4)[:, None, None] & 15)[..., :d] * c["v_scale"][page, :, slot][..., None]
    return tuple(torch.where(live, torch.matmul(x, hd), 0.0).to(dtype) for x in (k, v))


def _rotated(n, cos, sin, r, interleaved):
    """n [t, h, d], its first r channels rotated by cos, sin [t, 1, r / 2]."""
    a, b = (n[..., 0:r:2], n[..., 1:r:2]) if interleaved else (n[..., :r // 2], n[..., r // 2:r])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, n[..., r:]], -1)


def _append_plain(s):
    c, ps, d, r = s["cache"], s["page"], s["d"], s["rotary"]
    b, live, back = _places(s, s["most_new"])
    pos = torch.where(live, s["lengths"][b].long() - back, 0)
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]

    def head(x, w, wide):
        x = x.to(wide)
        if s["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(wide)
        return _rotated(x, cos.to(wide), sin.to(wide), r, s["interleaved"])

    q = torch.where(live[:, None, None], head(s["q"], s["q_weight"], torch.float32), 0.0).to(s["q"].dtype)
    hd = _hadamard(d, torch.float64)
    page, slot = s["page_table"][b, pos // ps].long(), pos % ps
    # tokens of no sequence are left out, by what is in the cache already
    code, scale = _codes(torch.matmul(head(s["k"], s["k_weight"], torch.float64), hd))
    at = live.nonzero()[:, 0]
    c["k"][page[at], :, slot[at], :d // 2] = (code[..., 0::2] | code[..., 1::2] << 4)[at]
    c["k_scale"][page[at], :, slot[at]] = scale[at]
    code, scale = _codes(torch.matmul(s["v"].double(), hd))
    c["v_scale"][page[at], :, slot[at]] = scale[at]
    for odd in (0, 1):                          # two tokens share a byte
        at = (live & (slot % 2 == odd)).nonzero()[:, 0]
        byte = c["v"].transpose(3, 4)
        where = (page[at], slice(None), slot[at] // 8, slot[at] % 8 // 2, slice(0, d))
        byte[where] = byte[where] & (15 if odd else 240) | code[at] << 4 * odd
    return (q,) + _read_plain(s, _stored(s))


def _attend_plain(s):
    c, ps, d, h, hk = s["cache"], s["page"], s["d"], s["heads"], s["kv_heads"]
    n, longest, batch = s["most_new"], s["longest"], s["batch"]
    hd = _hadamard(d, torch.float32)
    b, live, back = _places(s, n)
    # the queries as [batch, kv_heads, group x new tokens, d], each sequence's at the end
    at = torch.where(live, b * n + n - back, batch * n)
    q = torch.zeros((batch * n + 1, h, d), device="cuda")
    q[at] = torch.matmul(s["q"].float(), hd) * (1.0 / math.sqrt(d))
    q = q[:-1].view(batch, n, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(batch, hk, -1, d)
    # keys and values of the longest sequence's length, in the transformed basis
    groups = torch.arange(_ceil(longest, 8), device="cuda")
    page = s["page_table"][:, groups * 8 // ps].clamp(min=0).long()                          # [batch, groups]
    part = (groups % (ps // 8))[None].expand_as(page)
    k = c["k"].view(c["k"].shape[0], hk, ps // 8, 8, -1)[page, :, part]                      # [batch, groups, kv_heads, 8, pitch / 2]
    k = _numbers(_nibbles(k))[..., :d] * c["k_scale"].view(-1, hk, ps // 8, 8)[page, :, part][..., None]
    k = k.permute(0, 2, 1, 3, 4).reshape(batch, hk, -1, d)
    v = _numbers(_nibbles(c["v"][page, :, part]))[..., :d, :].transpose(3, 4)
    v = v * c["v_scale"].view(-1, hk, ps // 8, 8)[page, :, part][..., None]
    v = v.permute(0, 2, 1, 3, 4).reshape(batch, hk, -1, d)
    key = torch.arange(k.shape[2], device="cuda")
    pos = s["lengths"][:, None] - n + torch.arange(n, device="cuda")                         # [batch, n]
    seen = key <= pos[..., None]
    if s["window"]:
        seen &= (key > pos[..., None] - s["window"]) | (key < s["sinks"])
    seen = seen[:, None].expand(-1, h // hk, -1, -1).reshape(batch, 1, -1, key.numel())
    score = torch.matmul(q, k.transpose(2, 3))
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-37)
    out = torch.matmul(out, hd).view(batch, hk, h // hk, n, d).permute(0, 3, 1, 2, 4).reshape(batch * n, h, d)
    out = torch.cat([out, out.new_zeros((1, h, d))])
    return out[at].to(s["q"].dtype)


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "attend":
        return _attend_plain(s)
    return _append_plain(s) if s["op"] == "append" else _read_plain(s, _DTYPE[s["dtype"]])


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _walsh(x, block):
    """The transform of the last axis, step by step."""
    shape, step = x.shape, 1
    while step < block:
        x = x.reshape(shape[:-1] + (shape[-1] // (2 * step), 2, step))
        x = torch.stack([x[..., 0, :] + x[..., 1, :], x[..., 0, :] - x[..., 1, :]], -2).reshape(shape)
        step *= 2
    return x / math.sqrt(block)


def _e2m1(code):
    """The number of a code: one bit of sign, two of exponent, one of mantissa."""
    e, m = (code >> 1 & 3).double(), (code & 1).double()
    return torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e - 1)) * (1 - 2 * (code >> 3).double())


def _nearest(a):
    """a >= 0 to the nearest E2M1 number, ties to even."""
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.round(a / step) * step).clamp(max=6)


def _cached(s, b, length, head=None):
    """(k, v) [tokens, kv_heads, d] of a sequence, in the transformed basis; or of one head."""
    c, ps, d = s["cache"], s["page"], s["d"]
    page = s["page_table"][b, :_ceil(length, ps)].long()
    heads = slice(None) if head is None else slice(head, head + 1)
    k, v = c["k"][page][:, heads], c["v"][page][:, heads]                                    # [pages, heads, ..]
    k = torch.stack([_e2m1(k & 15), _e2m1(k >> 4)], -1).flatten(-2)[..., :d] * c["k_scale"][page][:, heads].double()[..., None]
    v = torch.stack([_e2m1(v & 15), _e2m1(v >> 4)], -1).flatten(-2)[..., :d, :].transpose(3, 4).flatten(2, 3)
    v = v * c["v_scale"][page][:, heads].double()[..., None]
    return tuple(x.transpose(1, 2).flatten(0, 1)[:length] for x in (k, v))


def exact(case, seed):
    s = prepare(case, seed)
    new, lengths = _sequences(case)
    h, hk, d, block = case["heads"], case["kv_heads"], case["d"], _block(case["d"])
    if case["op"] == "read":
        both = [_cached(s, b, n) for b, n in enumerate(lengths)]
        return tuple(_walsh(torch.cat([x[i] for x in both]), block) for i in (0, 1))
    if case["op"] == "append":
        t, r = s["t"], case["rotary"]
        pos = torch.cat([torch.arange(n - m, n) for m, n in zip(new, lengths)]).cuda()
        turn = torch.complex(s["cos"].double(), s["sin"].double())[pos][:, None]             # [t, 1, r / 2]
        rows = pos.numel()

        def turned(x, w):
            x = x[:rows].double()
            if case["norm"]:
                x = x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
            if case["interleaved"]:
                z = torch.complex(x[..., 0:r:2].contiguous(), x[..., 1:r:2].contiguous()) * turn
                y = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
                y = torch.cat([z.real, z.imag], -1)
            return torch.cat([y, x[..., r:]], -1)

        def stored(x):
            z = _walsh(x, block)
            top = z.abs().amax(-1, keepdim=True)
            scale = torch.where(top > 0, top / 6, 1.0)
            return _walsh(torch.sign(z) * _nearest(z.abs() / scale) * scale, block)

        padded = torch.zeros((t - rows, 1, d), dtype=torch.float64, device="cuda")
        return tuple(torch.cat([x, padded.expand(-1, x.shape[1], -1)]) for x in
                     (turned(s["q"], s["q_weight"]), stored(turned(s["k"], s["k_weight"])), stored(s["v"][:rows].double())))
    out = torch.zeros((s["t"], h, d), dtype=torch.float64, device="cuda")
    g, at = h // hk, 0
    for b, (m, n) in enumerate(zip(new, lengths)):
        i, j = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        hidden = j > i
        if case["window"]:
            hidden |= (j <= i - case["window"]) & (j >= case["sinks"])
        for head in range(hk):
            k, v = (x[:, 0] for x in _cached(s, b, n, head))
            for e in range(head * g, head * g + g):
                q = _walsh(s["q"][at:at + m, e].double(), block)
                w = torch.softmax((q @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf), -1)
                out[at:at + m, e] = _walsh(w @ v, block)
        at += m
    return out


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    size, h, hk, d = _SIZE[case["dtype"]], case["heads"], case["kv_heads"], case["d"]
    new, lengths = _sequences(case)
    t, token = _total(case), 2 * hk * (d // 2 + 4)          # bytes of a token in the cache
    steps = 2 * int(math.log2(_block(d)))
    if case["op"] == "read":
        return {"bytes": t * (token + 2 * hk * d * size), "flops": t * 2 * hk * d * steps}
    if case["op"] == "append":
        # q, k, v and the tables read, q and codes written, the stored values written
        return {"bytes": t * ((2 * h + 2 * hk) * d * size + token + 4 * hk * d) + 4 * case["rotary"] * sum(new),
                "flops": t * (8 * (h + hk) * d + 2 * hk * d * 2 * steps)}
    pairs = tokens = 0
    for m, n in zip(new, lengths):
        window, sinks = case["window"] or n, case["sinks"] if case["window"] else 0
        first = max(0, n - m + 1 - window)                  # the oldest token that the first query's window holds
        tokens += n - first + min(sinks, first)
        for i in range(n - m, n):
            low = max(0, i + 1 - window)
            pairs += i + 1 - low + min(sinks, low)
    return {"bytes": tokens * token + 2 * t * h * d * size, "flops": 4 * d * h * pairs}
