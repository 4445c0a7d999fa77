// Keys and values into a paged cache of 4-bit codes, on the way from the projection, and back out of it.
//
//     n = x r w,  r = (mean x^2 + eps)^-1/2   (queries and keys, where the call has a norm),   y = R(position) n
//     queries: y.   keys: z = H y.   values: z = H v.   scale = max |z| / 6,  code = E2M1(z / scale)
//
// H is orthonormal, symmetric, block-diagonal: its blocks spread a large channel over their width, so that one scale serves a head.  All in
// fp32; roundings: of the query to its type, of the scale, of the code.
//
// A workgroup takes the tokens of one group of 8 positions, because a dword of the cache's v holds the codes of a channel for 8 tokens: it
// is then written by one workgroup, whole where all 8 tokens are new, around what it held where they are not.  A head is owned by LP
// neighbouring lanes, 8 channels each; a lane keeps its token's cosines, sines and both channels' weights over all heads of the token.  The
// other channel of a pair comes from memory a second time (a cache line that the wave has just read) instead of through LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hq_common.h"
#include "hq_floats.h"
#include "hq_fp8.h"
#include "hq_kv4.h"
#include "hq_kv4_check.h"
#include "hq_kv4_lanes.h"

namespace {

// The group of tokens that a workgroup works on: every wave looks for the sequence by itself.
__device__ __forceinline__ hq::Kv4Group group_of(const hq::Kv4 &c, int index) {
    const int lane = threadIdx.x & 63;
    int s = -1;
    for (int base = 0; base <= c.batch; base += 64) {
        const int at = base + lane;
        const bool before = at <= c.batch && hq::kv4_group_begin(c.begin(at), at) <= index;
        s += __popcll(__ballot(before));
    }
    return hq::kv4_group(c, __builtin_amdgcn_readfirstlane(hq::kv4_max(s, 0)), index);
}

// ---- append -----------------------------------------------------------------------------------------------------------
struct AppendArgs {
    hq::Kv4 c;
    const void *q, *k, *v, *q_weight, *k_weight;
    void *q_out;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;   // strides, in elements
    const float *cos, *sin;   // [positions, rotary / 2]
    const void *pos;          // int32 or int64 per token, or null: the place in the sequence
    int64_t positions;
    int heads, rotary, pos_wide, interleaved, w_float, norm;
    float eps;
};

// What a lane does to each head of its token.
struct Turn {
    bool pad, beyond;
    float cos[8], sin[8];   // y = x cos + (the pair's other channel) sin
};
// The other channel of channel c's pair where pairs are halves of the rotated part apart; c itself for a channel that is not rotated.
__device__ __forceinline__ int partner_of(int c, int rotary) {
    const int half = rotary >> 1;
    return c < half ? c + half : c < rotary ? c - half : c;
}
__device__ __forceinline__ Turn turn_of(const AppendArgs &a, int row, int64_t place, int c0) {
    Turn t;
    int64_t p = place;
    if (a.pos) p = a.pos_wide ? static_cast<const int64_t *>(a.pos)[row] : static_cast<const int32_t *>(a.pos)[row];
    t.pad = p < 0 || place < 0;
    t.beyond = !t.pad && a.rotary && p >= a.positions;
    const int half = a.rotary >> 1;
    const int64_t at = (t.pad || t.beyond ? 0 : p) * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        t.cos[i] = 1.0f;
        t.sin[i] = 0.0f;
        if (c < a.rotary) {
            const int pair = a.interleaved ? c >> 1 : c < half ? c : c - half;
            const bool first = a.interleaved ? !(c & 1) : c < half;
            t.cos[i] = a.cos[at + pair];
            const float s = a.sin[at + pair];
            t.sin[i] = first ? -s : s;
        }
    }
    return t;
}
// A lane's 8 channels as they are, and those of their pairs' other channels.  QUADS: runs of 4 channels have theirs in runs of 4.
template <class T, bool QUADS>
__device__ __forceinline__ void load_partners(const T *x, int c0, int rotary, float (&v)[8]) {
    if constexpr (QUADS) {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const typename Vec<T, 4>::type t = load_vec<T, 4>(x + partner_of(c0 + i, rotary));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i + e] = static_cast<float>(t[e]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(x[partner_of(c0 + i, rotary)]);
    }
}
template <class T, bool QUADS>
__device__ __forceinline__ void weights_of(const AppendArgs &a, const void *w, int c0, float (&own)[8], float (&other)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) own[i] = other[i] = 1.0f;
    if (!w) return;
    if (a.w_float) {
        load8(static_cast<const float *>(w) + c0, own);
        if (!a.interleaved) load_partners<float, QUADS>(static_cast<const float *>(w), c0, a.rotary, other);
    } else {
        load8(static_cast<const T *>(w) + c0, own);
        if (!a.interleaved) load_partners<T, QUADS>(static_cast<const T *>(w), c0, a.rotary, other);
    }
}
// A head normalised and turned.
template <class T, int LP, bool QUADS>
__device__ __forceinline__ void head(const AppendArgs &a, const T *x, int c0, bool live, const Turn &t, const float (&own)[8],
                                     const float (&other)[8], float (&v)[8]) {
    float p[8];
    load8(x + c0, v);
    if (!a.interleaved && a.rotary) load_partners<T, QUADS>(x, c0, a.rotary, p);
    float r = 1.0f;
    if (a.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i] * v[i];
        sum = sum_lanes<LP>(live ? sum : 0.0f);
        r = 1.0f / sqrtf(sum * (1.0f / static_cast<float>(a.c.d)) + a.eps);
    }
    if (t.beyond) r = __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= r * own[i];
    if (!a.rotary) return;
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = v[i ^ 1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] *= r * other[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c0 + i < a.rotary) v[i] = v[i] * t.cos[i] + p[i] * t.sin[i];
}
// Its transform in codes.
template <int LP>
__device__ __forceinline__ uint32_t coded(float (&v)[8], int in, bool live, int block_log2, float &scale) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = live ? v[i] : 0.0f;
    walsh(v, in, block_log2);
    const float f = walsh_factor(block_log2);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] *= f;
        top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    scale = kv4_scale(max_lanes<LP>(top));
    return kv4_codes(v, scale == scale ? __fdiv_rn(1.0f, scale) : 0.0f);
}

template <int DT, int LP, bool QUADS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    using T = typename Float<DT>::type;
    constexpr int SLOTS = 256 / LP;
    const hq::Kv4Group g = group_of(a.c, blockIdx.x);
    if (g.count == 0) return;
    // slots: tokens, a power of two of them, times heads at once
    const int log2 = g.count > 4 ? 3 : g.count > 2 ? 2 : g.count - 1, at_once = SLOTS >> log2;
    const int in = threadIdx.x % LP, slot = threadIdx.x / LP, token = slot & ((1 << log2) - 1), first = slot >> log2;
    const bool live = in * 8 < a.c.d, mine = token < g.count;
    const int c0 = live ? in * 8 : 0, row = g.row + (mine ? token : 0);
    const int64_t place = g.s < a.c.batch ? g.position + (mine ? token : 0) : -1;
    const Turn turn = turn_of(a, row, place, c0);
    const int part = blockIdx.y, parts = gridDim.y;
    float own[8], other[8], x[8];
    weights_of<T, QUADS>(a, a.q_weight, c0, own, other);
    for (int h = part * at_once + first; h < a.heads; h += parts * at_once) {
        const T *q = static_cast<const T *>(a.q) + row * a.q_token + h * a.q_head;
        head<T, LP, QUADS>(a, q, c0, live, turn, own, other, x);
        if (turn.pad) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        }
        if (live && mine) store8(static_cast<T *>(a.q_out) + row * a.out_token + h * a.out_head + c0, x);
    }
    if (g.s >= a.c.batch) return;
    // (positions of a group of 8 are all negative, without a page, or none is)
    const int64_t page = a.c.page(g.s, g.position);
    if (page < 0) return;
    const bool stored = mine && !turn.pad;
    weights_of<T, QUADS>(a, a.k_weight, c0, own, other);
    for (int h = part * at_once + first; h < a.c.kv_heads; h += parts * at_once) {
        const T *k = static_cast<const T *>(a.k) + row * a.k_token + h * a.k_head;
        head<T, LP, QUADS>(a, k, c0, live, turn, own, other, x);
        float scale;
        const uint32_t w = coded<LP>(x, in, live, a.c.block_log2, scale);
        if (!stored) continue;
        const int64_t at = a.c.slots(page, h) + a.c.slot(static_cast<int>(place));
        if (live) *reinterpret_cast<uint32_t *>(a.c.k + at * a.c.row_bytes() + in * 4) = w;
        if (in == 0) a.c.k_scale[at] = scale;
    }
    __shared__ uint32_t codes[SLOTS][LP + 1];
    __shared__ uint32_t new_tokens;   // four bits for each token of the group that is stored
    if (threadIdx.x == 0) new_tokens = 0;
    __syncthreads();
    if (first == 0 && in == 0 && stored) atomicOr(&new_tokens, 15u << (4 * (static_cast<int>(place) & 7)));
    for (int base = part * at_once; base < a.c.kv_heads; base += parts * at_once) {
        const int h = base + first;
        if (h < a.c.kv_heads) {
            load8(static_cast<const T *>(a.v) + row * a.v_token + h * a.v_head + c0, x);
            float scale;
            codes[slot][in] = coded<LP>(x, in, live, a.c.block_log2, scale);
            if (stored && in == 0) a.c.v_scale[a.c.slots(page, h) + a.c.slot(static_cast<int>(place))] = scale;
        }
        __syncthreads();
        const uint32_t mask = new_tokens;
        const int skip = g.position & 7, ahead = g.position & ~7;
        for (int e = threadIdx.x; e < at_once * a.c.d; e += 256) {
            const int local = e / a.c.d, c = e - local * a.c.d;
            if (base + local >= a.c.kv_heads) break;
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int from = i - skip;
                if (from >= 0 && from < g.count) w |= (codes[(local << log2) + from][c >> 3] >> (4 * (c & 7)) & 15u) << (4 * i);
            }
            uint32_t *to = reinterpret_cast<uint32_t *>(a.c.v + (a.c.slots(page, base + local) + a.c.slot(ahead)) * a.c.row_bytes()) + c;
            if (mask != 0xFFFFFFFFu) w = (w & mask) | (*to & ~mask);
            if (mask) *to = w;
        }
        __syncthreads();
    }
}

// ---- read -------------------------------------------------------------------------------------------------------------
struct ReadArgs {
    hq::Kv4 c;
    void *k, *v;   // [t, kv_heads, d], dense
};

template <int DT, int LP>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
    using T = typename Float<DT>::type;
    constexpr int SLOTS = 256 / LP;
    const hq::Kv4Group g = group_of(a.c, blockIdx.x);
    if (g.count == 0) return;
    const int log2 = g.count > 4 ? 3 : g.count > 2 ? 2 : g.count - 1, at_once = SLOTS >> log2;
    const int in = threadIdx.x % LP, slot = threadIdx.x / LP, token = slot & ((1 << log2) - 1), first = slot >> log2;
    const bool live = in * 8 < a.c.d && token < g.count;
    const int row = g.row + token, place = g.s < a.c.batch ? g.position + token : -1;
    const int64_t page = g.s < a.c.batch ? a.c.page(g.s, g.position) : -1;
    const float factor = walsh_factor(a.c.block_log2), nothing = place < 0 ? 0.0f : __builtin_nanf("");
    const int ahead = g.position & ~7;
    __shared__ uint32_t codes[256];   // v's dwords of one turn: [heads at once, d]
    for (int base = blockIdx.y * at_once; base < a.c.kv_heads; base += gridDim.y * at_once) {
        const int h = base + first;
        const bool mine = live && h < a.c.kv_heads;
        for (int v = 0; v < 2; ++v) {
            float x[8];
            float scale = 0.0f;
            uint32_t w = 0;
            const int64_t at = page < 0 || place < 0 || !mine ? 0 : a.c.slots(page, h) + a.c.slot(place);
            if (mine && page >= 0 && place >= 0) scale = (v ? a.c.v_scale : a.c.k_scale)[at];
            if (v == 0) {
                if (mine && page >= 0 && place >= 0) w = *reinterpret_cast<const uint32_t *>(a.c.k + at * a.c.row_bytes() + in * 4);
            } else {
                for (int part = 0; part < at_once * a.c.d; part += 256) {
                    const int e = part + threadIdx.x, local = e / a.c.d, c = e - local * a.c.d;
                    __syncthreads();
                    if (e < at_once * a.c.d && base + local < a.c.kv_heads && page >= 0)
                        codes[threadIdx.x] =
                            *(reinterpret_cast<const uint32_t *>(a.c.v + (a.c.slots(page, base + local) + a.c.slot(ahead)) * a.c.row_bytes()) + c);
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int from = first * a.c.d + in * 8 + i - part;
                        if (mine && page >= 0 && from >= 0 && from < 256) w |= (codes[from] >> (4 * (place & 7)) & 15u) << (4 * i);
                    }
                }
            }
            const half8v n = kv4_halves(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(n[i]);
            walsh(x, in, a.c.block_log2);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = page < 0 || place < 0 ? nothing : x[i] * (scale * factor);
            if (mine) store8(static_cast<T *>(v ? a.v : a.k) + (static_cast<int64_t>(row) * a.c.kv_heads + h) * a.c.d + in * 8, x);
        }
    }
}

// Workgroups beside each other share a group's heads where there are few groups.
uint32_t parts_for(int groups, int most, int lanes) {
    const int turns = std::max(1, (most + 256 / lanes / 8 - 1) / (256 / lanes / 8));
    const int wanted = (4 * hq::compute_units() + groups - 1) / groups;
    return static_cast<uint32_t>(std::max(1, std::min({wanted, turns, 64})));
}

template <int DT>
void launch_append(const AppendArgs &a, hipStream_t st) {
    const int groups = hq::kv4_groups(a.c.t, a.c.batch);
    const bool quads = (a.rotary >> 1) % 4 == 0;
    const auto go = [&](auto lp) {
        constexpr int LP = decltype(lp)::value;
        const dim3 grid(groups, parts_for(groups, std::max(a.heads, a.c.kv_heads), LP));
        if (quads) append_kernel<DT, LP, true><<<grid, 256, 0, st>>>(a);
        else append_kernel<DT, LP, false><<<grid, 256, 0, st>>>(a);
    };
    if (a.c.d <= 32) go(std::integral_constant<int, 4>{});
    else if (a.c.d <= 64) go(std::integral_constant<int, 8>{});
    else if (a.c.d <= 128) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 32>{});
}
template <int DT>
void launch_read(const ReadArgs &a, hipStream_t st) {
    const int groups = hq::kv4_groups(a.c.t, a.c.batch);
    const auto go = [&](auto lp) {
        constexpr int LP = decltype(lp)::value;
        read_kernel<DT, LP><<<dim3(groups, parts_for(groups, a.c.kv_heads, LP)), 256, 0, st>>>(a);
    };
    if (a.c.d <= 32) go(std::integral_constant<int, 4>{});
    else if (a.c.d <= 64) go(std::integral_constant<int, 8>{});
    else if (a.c.d <= 128) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 32>{});
}

}  // namespace

extern "C" hq_status hq_kv4_append(const hq_kv4 *cache, const void *q, const void *k, const void *v, hq_dtype dtype, int heads,
                                   const int64_t *strides, const void *q_weight, const void *k_weight, hq_dtype w_dtype, const float *cos,
                                   const float *sin, int64_t positions, int rotary, int interleaved, const void *pos, int pos_size, int norm,
                                   float eps, void *q_out, void *stream) {
    if (!cache || !strides || (rotary > 0 && (!cos || !sin))) return HQ_ERR_NULL;
    if (!hq::is_float(dtype) || (w_dtype != dtype && w_dtype != HQ_F32)) return HQ_ERR_DTYPE;
    hq::Kv4 c;
    if (const hq_status s = hq::kv4_check(*cache, heads, &c)) return s;
    if (c.t > 0 && (!q || !k || !v || !q_out)) return HQ_ERR_NULL;
    if (rotary < 0 || rotary > c.d || (rotary & 1) || (rotary && positions <= 0) || (norm && !(eps >= 0.0f))) return HQ_ERR_SHAPE;
    if (!norm && (q_weight || k_weight)) return HQ_ERR_SHAPE;
    if (pos && pos_size != 4 && pos_size != 8) return HQ_ERR_DTYPE;
    const int size = hq::size_of(dtype);
    for (const void *p : {q, k, v, static_cast<const void *>(q_out)})
        if (!hq::aligned_to(p, size)) return HQ_ERR_ALIGN;
    for (const void *p : {q_weight, k_weight})
        if (!hq::aligned_to(p, hq::size_of(w_dtype))) return HQ_ERR_ALIGN;
    if (!hq::aligned_to(cos, 4) || !hq::aligned_to(sin, 4) || !hq::aligned_to(pos, pos_size == 8 ? 8 : 4)) return HQ_ERR_ALIGN;
    if (c.t == 0) return HQ_OK;
    const AppendArgs a{c, q, k, v, q_weight, k_weight, q_out, strides[0], strides[1], strides[2], strides[3], strides[4], strides[5],
                       strides[6], strides[7], cos, sin, pos, positions, heads, rotary, pos_size == 8, interleaved != 0, w_dtype == HQ_F32,
                       norm != 0, eps};
    const hq::LaunchCheck check;
    const auto st = static_cast<hipStream_t>(stream);
    switch (dtype) {
        case HQ_F16: launch_append<HQ_F16>(a, st); break;
        case HQ_BF16: launch_append<HQ_BF16>(a, st); break;
        default: launch_append<HQ_F32>(a, st); break;
    }
    return check.status();
}

extern "C" hq_status hq_kv4_read(const hq_kv4 *cache, void *k, void *v, hq_dtype dtype, void *stream) {
    if (!cache) return HQ_ERR_NULL;
    if (!hq::is_float(dtype)) return HQ_ERR_DTYPE;
    hq::Kv4 c;
    if (const hq_status s = hq::kv4_check(*cache, cache->kv_heads, &c)) return s;
    if (c.t > 0 && (!k || !v)) return HQ_ERR_NULL;
    if (!hq::aligned_to(k, hq::size_of(dtype)) || !hq::aligned_to(v, hq::size_of(dtype))) return HQ_ERR_ALIGN;
    if (c.t == 0) return HQ_OK;
    const ReadArgs a{c, k, v};
    const hq::LaunchCheck check;
    const auto st = static_cast<hipStream_t>(stream);
    switch (dtype) {
        case HQ_F16: launch_read<HQ_F16>(a, st); break;
        case HQ_BF16: launch_read<HQ_BF16>(a, st); break;
        default: launch_read<HQ_F32>(a, st); break;
    }
    return check.status();
}
