// Keys and values into a paged cache of 4-bit codes, on the way from the projection, and back out of it.
//
//     n = x r w,  r = (mean x^2 + eps)^-1/2   (queries and keys, where the call has a norm),   y = R(position) n
//     queries: y.   keys: z = H y.   values: z = H v.   scale = max |z| / 6,  code = E2M1(6 z / max |z|)
//
// H is orthonormal, symmetric, block-diagonal: its blocks spread a large channel over their width, so that one scale serves a head.
// Queries and scales in fp32; roundings: of the query to its type, of the scale, of the code.  A code is the definition's: a head with a number
// closer to a border between two codes than its fp32 steps can be off is worked out in 64 bits (coded).
//
// A workgroup takes the tokens of one group of 8 positions, because a dword of the cache's v holds the codes of a channel for 8 tokens: it
// is then written by one workgroup, whole where all 8 tokens are new, around what it held where they are not.  A head is owned by LP
// neighbouring lanes, 8 channels each; a lane keeps its token's cosines, sines and weights over all heads of the token.  The other
// channel of a pair is in the lane, or in a lane that one permute reaches, or comes from memory a second time (a cache line that
// the wave has just read).
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

// What a caller's arrays on the device hold, by scalar loads: they are not written while a call runs.
__device__ __forceinline__ int32_t constant(const int32_t *p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uint64_t>(p));
}
// The group of tokens that a workgroup works on: every wave looks for the sequence by itself.
__device__ __forceinline__ hq::Kv4Group group_of(const hq::Kv4 &c, int index) {
    const auto length = [](const int32_t *p) { return constant(p); };
    if (!c.begins) {
        const int s = hq::kv4_sequence(c, index);
        return hq::kv4_group(c, s, c.begin(s), c.begin(s + 1), index, length);
    }
    const int lane = threadIdx.x & 63;
    int s = -1, mine = 0;
    for (int base = 0; base <= c.batch; base += 64) {
        const int at = base + lane;
        mine = at <= c.batch ? c.begin(at) : 0;
        s += __popcll(__ballot(at <= c.batch && hq::kv4_group_begin(mine, at) <= index));
    }
    s = __builtin_amdgcn_readfirstlane(hq::kv4_max(s, 0));
    if (c.batch < 64)   // (they are in the lanes)
        return hq::kv4_group(c, s, __builtin_amdgcn_readlane(mine, s), __builtin_amdgcn_readlane(mine, hq::kv4_min(s + 1, c.batch)), index, length);
    return hq::kv4_group(c, s, c.begin(s), c.begin(hq::kv4_min(s + 1, c.batch)), index, length);
}
__device__ __forceinline__ int64_t page_of(const hq::Kv4 &c, const hq::Kv4Group &g) {
    if (g.s >= c.batch) return -1;
    const int32_t *const table = c.table + static_cast<int64_t>(g.s) * c.table_pages;
    return c.checked(g.position, [&](int column) { return constant(table + column); });
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
    hq::Magic31 d_magic, part_magic;
    int q_parts, k_parts;
};

// Where the other channel of a pair is.
enum Pairs {
    kNeighbours,   // in the lane (or nothing is rotated)
    kLanes,        // in a lane whose block of channels differs in one bit: halves of 8, 16, 32 or 64 channels
    kQuads,        // in memory: runs of 4 channels have theirs in runs of 4
    kSingle        // in memory, one by one
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
template <int PAIRS>
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
        t.cos[i] = 1.0f;
        t.sin[i] = 0.0f;
    }
    // runs of channels with neighbouring pairs in one load
    constexpr int RUN = PAIRS == kLanes ? 8 : PAIRS == kSingle ? 1 : 4;
#pragma unroll
    for (int i = 0; i < 8; i += RUN) {
        const int c = c0 + i;
        if constexpr (PAIRS == kNeighbours) {
            // (channels 2 j and 2 j + 1 of a run of 4; the rotated part ends at an even one)
#pragma unroll
            for (int e = 0; e < 4; e += 2)
                if (c + e < a.rotary) {
                    const float x = a.cos[at + ((c + e) >> 1)], y = a.sin[at + ((c + e) >> 1)];
                    t.cos[i + e] = t.cos[i + e + 1] = x;
                    t.sin[i + e] = -y;
                    t.sin[i + e + 1] = y;
                }
        } else if (c < a.rotary) {
            const bool first = c < half;
            const int64_t from = at + (first ? c : c - half);
            const typename Vec<float, RUN>::type x = load_vec<float, RUN>(a.cos + from), y = load_vec<float, RUN>(a.sin + from);
#pragma unroll
            for (int e = 0; e < RUN; ++e) {
                t.cos[i + e] = x[e];
                t.sin[i + e] = first ? -y[e] : y[e];
            }
        }
    }
    return t;
}
// A lane's 8 channels of a head, and those of their pairs' other channels where these come from memory.
template <class T, int PAIRS> struct Raw {
    typename Vec<T, 8>::type v;
    T p[PAIRS >= kQuads ? 8 : 1];
    __device__ __forceinline__ void load(const T *x, int c0, int rotary) {
        v = load_vec<T, 8>(x + c0);
        if constexpr (PAIRS == kQuads) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const typename Vec<T, 4>::type t = load_vec<T, 4>(x + partner_of(c0 + i, rotary));
#pragma unroll
                for (int e = 0; e < 4; ++e) p[i + e] = t[e];
            }
        } else if constexpr (PAIRS == kSingle) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[partner_of(c0 + i, rotary)];
        }
    }
};
template <class T, int PAIRS>
__device__ __forceinline__ Raw<float, PAIRS> weights_of(const AppendArgs &a, const void *w, int c0) {
    Raw<float, PAIRS> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = 1.0f;
#pragma unroll
    for (float &x : r.p) x = 1.0f;
    if (!w) return r;
    if (a.w_float) {
        r.load(static_cast<const float *>(w), c0, a.rotary);
    } else {
        Raw<T, PAIRS> t;
        t.load(static_cast<const T *>(w), c0, a.rotary);
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = static_cast<float>(t.v[i]);
        if constexpr (PAIRS >= kQuads) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.p[i] = static_cast<float>(t.p[i]);
        }
    }
    return r;
}
// A head normalised and turned.
template <class T, int LP, int PAIRS>
__device__ __forceinline__ void head(const AppendArgs &a, const Raw<T, PAIRS> &x, int c0, bool live, const Turn &t, const Raw<float, PAIRS> &w,
                                     float (&v)[8]) {
    float r = 1.0f;
    if (a.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += static_cast<float>(x.v[i]) * static_cast<float>(x.v[i]);
        sum = sum_lanes<LP>(live ? sum : 0.0f) * (1.0f / static_cast<float>(a.c.d)) + a.eps;
        r = __builtin_amdgcn_rsqf(sum);                       // (off by one step at most)
        if (sum < 0x1p-120f) r = 1.0f / sqrtf(sum);           // (which it takes for 0 where it is not a normal number)
    }
    if (t.beyond) r = __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(x.v[i]) * (r * w.v[i]);
    if (!a.rotary) return;
    if constexpr (PAIRS == kLanes) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[i] * t.cos[i];
        const int half = a.rotary >> 4;   // in blocks
        if (half == 8) add_lanes<3>(y, v, t.sin);
        else if (half == 4) add_lanes<2>(y, v, t.sin);
        else if (half == 2) add_lanes<1>(y, v, t.sin);
        else add_lanes<0>(y, v, t.sin);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c0 < a.rotary ? y[i] : v[i];
    } else {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kNeighbours) p[i] = v[i ^ 1];
            else p[i] = static_cast<float>(x.p[i]) * (r * w.p[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c0 + i < a.rotary) v[i] = v[i] * t.cos[i] + p[i] * t.sin[i];
    }
}
// The length of a head before weights and norm.
template <class T, int LP, int PAIRS>
__device__ __forceinline__ float length_of(const Raw<T, PAIRS> &x, bool live) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += static_cast<float>(x.v[i]) * static_cast<float>(x.v[i]);
    return __builtin_amdgcn_sqrtf(sum_lanes<LP>(live ? sum : 0.0f));
}
// Its number in 64 bits, where it is used: what is the same for all heads is not to be converted ahead of them, into registers.
__device__ __forceinline__ double here(float x) {
    asm volatile("" : "+v"(x));
    return x;
}
// A head in 64 bits without the norm's factor, which all of its channels share.
template <class T, int PAIRS>
__device__ __forceinline__ void head_wide(const AppendArgs &a, const Raw<T, PAIRS> &x, int c0, const Turn &t, const Raw<float, PAIRS> &w,
                                          double (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<double>(x.v[i]) * here(w.v[i]);
    if (!a.rotary) return;
    double p[8];
    if constexpr (PAIRS == kLanes) {
        const int half = a.rotary >> 4;   // in blocks
        if (half == 8) other_lanes_wide<3>(v, p);
        else if (half == 4) other_lanes_wide<2>(v, p);
        else if (half == 2) other_lanes_wide<1>(v, p);
        else other_lanes_wide<0>(v, p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kNeighbours) p[i] = v[i ^ 1];
            else p[i] = static_cast<double>(x.p[i]) * here(w.p[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c0 + i < a.rotary) v[i] = v[i] * here(t.cos[i]) + p[i] * here(t.sin[i]);
}
// The norm's factor.
template <class T, int LP, int PAIRS>
__device__ __forceinline__ double norm_wide(const AppendArgs &a, const Raw<T, PAIRS> &x, bool live) {
    if (!a.norm) return 1.0;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += static_cast<double>(x.v[i]) * static_cast<double>(x.v[i]);
    sum = reduce_wide<LP>(live ? sum : 0.0, [](double a, double b) { return a + b; });
    return 1.0 / sqrt(sum / a.c.d + a.eps);
}
// A head's transform in codes by fp32 steps (the lanes without channels have zeros), and whether these leave one of its codes uncertain:
// `near`.  With u = 2^-24 and E at least the sum of the head's magnitudes before they are turned, each times |cos| + |sin| of its pair:
// products and the turn are off by 4 u E at most over a block (none for values), the steps of the transform by 6 u E and u of the result,
// which with the same error of the largest is 12 (4 + 6) u E / max of a number up to 6, and 12 u; the largest, the scale, its inverse (two),
// the factor and the product: 6 u of it.  Uncertain are codes of which the number less and plus that differ: those of 1 or 2 heads of 128
// normal values in 100.  ROUNDINGS: 4 + 6 for keys, 6 for values, with room for terms of second order.
template <int LP, int ROUNDINGS>
__device__ __forceinline__ uint32_t coded(float (&v)[8], float size, int in, int block_log2, float &scale, bool &near) {
    walsh_of<LP>(v, in, block_log2);
    const float f = walsh_factor(in, block_log2);
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits = max(bits, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const float top = __uint_as_float(max_lanes<LP>(bits)) * fabsf(f);
    scale = kv4_scale(top);
    const bool none = !(top > 0.0f && top < __builtin_inff());   // (codes of 0)
    const float by = f * __builtin_amdgcn_rcpf(scale), off = fmaf(size * fabsf(by), 2.02f * ROUNDINGS * 0x1p-24f, 52 * 0x1p-24f);
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = fmaf(v[i], by, off);
    const uint32_t w = kv4_codes(t);
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = fmaf(v[i], by, -off);
    // (the signs of a 0 may differ; next to the ends of fp32 a step, or a square, can be off by more than u)
    near = !none && (((w ^ kv4_codes(t)) & 0x77777777u) || !(off < 0.125f) || !(top > 0x1p-50f && top < 0x1p100f));
    return none ? 0u : w;
}
// The codes of such a head from what goes into the transform in 64 bits, times r.
template <int LP>
__device__ __forceinline__ uint32_t coded_wide(double (&v)[8], int in, bool live, int block_log2, double r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = live ? v[i] : 0.0;
    walsh_wide(v, in, block_log2);
    // (the least scale is 2^-126: the largest counts as 6 times that, in units of the sums)
    return kv4_codes_wide<LP>(v, __builtin_ldexp(block_log2 & 1 ? 1.4142135623730951 : 1.0, (block_log2 >> 1) - 126) * 6.0 / r);
}
// Whether any of the head's lanes says so.
template <int LP>
__device__ __forceinline__ bool any_of_head(uint64_t lanes) {
    return lanes >> (threadIdx.x & (64 - LP)) & ((uint64_t{1} << LP) - 1);
}

constexpr int kAtOnce = 4;   // heads of a slot whose loads are under way together

// The heads of a slot's token from head `from` on, `step` apart, below `heads`: queries go out, keys into the cache.
template <class T, int LP, int PAIRS, bool KEYS>
__device__ __forceinline__ void turned_heads(const AppendArgs &a, int from, int step, int heads, int row, int64_t place, int in, bool live, bool mine,
                                             const hq::Kv4Group &g) {
    // (positions of a group of 8 are all negative, without a page, or none is)
    const int64_t page = KEYS ? page_of(a.c, g) : 0;
    if (page < 0) return;
    const int c0 = live ? in * 8 : 0;
    const int64_t by_head = KEYS ? a.k_head : a.q_head;
    const T *x = static_cast<const T *>(KEYS ? a.k : a.q) + row * (KEYS ? a.k_token : a.q_token) + from * by_head;
    const int64_t x_step = step * by_head;
    if constexpr (!KEYS) {
        Raw<T, PAIRS> raw[kAtOnce];
        const auto load = [&](int h) {
#pragma unroll
            for (int e = 0; e < kAtOnce; ++e) {
                if (h + e * step < heads) raw[e].load(x, c0, a.rotary);
                x += x_step;
            }
        };
        load(from);
        const Raw<float, PAIRS> w = weights_of<T, PAIRS>(a, a.q_weight, c0);
        const Turn turn = turn_of<PAIRS>(a, row, place, c0);
        T *out = static_cast<T *>(a.q_out) + row * a.out_token + from * a.out_head + c0;
        for (int h = from; h < heads; h += kAtOnce * step) {
#pragma unroll
            for (int e = 0; e < kAtOnce; ++e) {
                if (h + e * step >= heads) break;
                float v[8];
                head<T, LP, PAIRS>(a, raw[e], c0, live, turn, w, v);
                if (__any(turn.pad)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = turn.pad ? 0.0f : v[i];
                }
                if (live && mine) store8(out, v);
                out += step * a.out_head;
            }
            load(h + kAtOnce * step);
        }
    } else {
        // (one head ahead: four at once, as queries, with the heads in 64 bits beside them cost a wave a SIMD, 182 us for 168 at best)
        Raw<T, PAIRS> next;
        if (from < heads) next.load(x, c0, a.rotary);
        Raw<float, PAIRS> w = weights_of<T, PAIRS>(a, a.k_weight, c0);
        Turn turn = turn_of<PAIRS>(a, row, place, c0);
        // E by lengths: that of x (d^1/2 with a norm) times that of the weights, each times |cos| + |sin|.  Lanes without channels have zeros.
        float size = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w.v[i] = live ? w.v[i] : 0.0f;
            turn.sin[i] = live ? turn.sin[i] : 0.0f;
            const float y = w.v[i] * (fabsf(turn.cos[i]) + fabsf(turn.sin[i]));
            size = fmaf(y, y, size);
        }
        size = sqrtf(sum_lanes<LP>(size) * (a.norm ? static_cast<float>(a.c.d) : 1.0f));
        if (a.norm && a.eps < 0x1p-110f) size *= 2.0f;   // (squares that are no normal numbers make the norm's factor up to 1.3 times too large)
        const int64_t at = a.c.slots(page, from) + a.c.slot(static_cast<int>(place)), scale_step = static_cast<int64_t>(step) << a.c.page_log2;
        uint8_t *code_out = a.c.k + at * a.c.row_bytes() + in * 4;
        float *scale_out = a.c.k_scale + at;
        uint32_t again = 0;
        for (int h = from; h < heads; h += step) {
            const Raw<T, PAIRS> now = next;
            x += x_step;
            if (h + step < heads) next.load(x, c0, a.rotary);
            float v[8], scale, most = size;
            if (!a.norm) most *= length_of<T, LP>(now, live);
            head<T, LP, PAIRS>(a, now, c0, live, turn, w, v);
            bool near;
            uint32_t code = coded<LP, 10>(v, most, in, a.c.block_log2, scale, near);
            again = again << 1 | (again & 0x80000000u);
            if (const uint64_t lanes = __ballot(near)) again |= any_of_head<LP>(lanes);
            if (mine && !turn.pad) {
                if (live) *reinterpret_cast<uint32_t *>(code_out) = code;
                if (in == 0) *scale_out = scale;
            }
            code_out += scale_step * a.c.row_bytes();
            scale_out += scale_step;
        }
        // The uncertain heads, the last one in bit 0, any before the last 31 in bit 31: a loop of its own, from memory again, so that it costs
        // no registers above.
        if (again)
            for (int h = from + (heads - 1 - from) / step * step, back = 0; h >= from; h -= step, back = hq::kv4_min(back + 1, 31))
                if (again >> back & 1) {
                    Raw<T, PAIRS> one;
                    one.load(static_cast<const T *>(a.k) + row * a.k_token + h * a.k_head, c0, a.rotary);
                    const double factor = norm_wide<T, LP>(a, one, live);
                    double v[8];
                    head_wide(a, one, c0, turn, w, v);
                    const uint32_t code = coded_wide<LP>(v, in, live, a.c.block_log2, factor);
                    uint8_t *const to = a.c.k + (a.c.slots(page, h) + a.c.slot(static_cast<int>(place))) * a.c.row_bytes() + in * 4;
                    if (mine && live && !turn.pad) *reinterpret_cast<uint32_t *>(to) = code;
                }
    }
}

// The values of a group's tokens, likewise.
template <class T, int LP>
__device__ __forceinline__ void stored_heads(const AppendArgs &a, int part, int log2, int at_once, int slot, int first, int row, int64_t place,
                                             int in, bool live, bool mine, const hq::Kv4Group &g) {
    constexpr int SLOTS = 256 / LP;
    const int parts = a.k_parts;
    const int64_t page = page_of(a.c, g);
    if (page < 0) return;
    const int c0 = live ? in * 8 : 0;
    __shared__ uint32_t codes[SLOTS][LP + 1];
    __shared__ uint32_t new_tokens;   // four bits for each token of the group that is stored
    if (threadIdx.x == 0) new_tokens = 0;
    bool stored = mine;
    if (a.pos && (a.pos_wide ? static_cast<const int64_t *>(a.pos)[row] : static_cast<const int32_t *>(a.pos)[row]) < 0) stored = false;
    const T *x = static_cast<const T *>(a.v) + row * a.v_token + c0;
    const int64_t at = a.c.slots(page, 0);
    float next[8];
    if (part * at_once + first < a.c.kv_heads) load8(x + (part * at_once + first) * a.v_head, next);
    __syncthreads();
    if (first == 0 && in == 0 && stored) atomicOr(&new_tokens, 15u << (4 * (static_cast<int>(place) & 7)));
    for (int base = part * at_once; base < a.c.kv_heads; base += parts * at_once) {
        const int h = base + first;
        if (h < a.c.kv_heads) {
            float v[8], scale, size = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = live ? next[i] : 0.0f;
                size += fabsf(v[i]);
            }
            if (h + parts * at_once < a.c.kv_heads) load8(x + (h + parts * at_once) * a.v_head, next);
            bool near;
            uint32_t code = coded<LP, 6>(v, sum_lanes<LP>(size), in, a.c.block_log2, scale, near);
            if (const uint64_t lanes = __ballot(near)) {
                load8(x + h * a.v_head, v);   // (again: no registers for it above)
                double wide[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) wide[i] = v[i];
                const uint32_t exact = coded_wide<LP>(wide, in, live, a.c.block_log2, 1.0);
                if (any_of_head<LP>(lanes)) code = exact;
            }
            codes[slot][in] = code;
            if (stored && in == 0) a.c.v_scale[at + (static_cast<int64_t>(h) << a.c.page_log2) + a.c.slot(static_cast<int>(place))] = scale;
        }
        __syncthreads();
        const uint32_t mask = new_tokens;
        const int skip = g.position & 7, ahead = a.c.slot(g.position & ~7);
        for (int e = threadIdx.x; e < at_once * a.c.d; e += 256) {
            const int local = hq::div_magic31(e, a.c.d, a.d_magic.m, a.d_magic.s), c = e - local * a.c.d;
            if (base + local >= a.c.kv_heads) break;
            uint32_t *to = reinterpret_cast<uint32_t *>(a.c.v + (at + (static_cast<int64_t>(base + local) << a.c.page_log2) + ahead) * a.c.row_bytes()) + c;
            uint32_t w = 0;
            if (mask != 0xFFFFFFFFu) w = *to & ~mask;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int from = i - skip;
                if (from >= 0 && from < g.count && (mask >> (4 * i) & 1)) w |= (codes[(local << log2) + from][c >> 3] >> (4 * (c & 7)) & 15u) << (4 * i);
            }
            if (mask) *to = w;
        }
        __syncthreads();
    }
}

// Workgroups of a group, side by side: q_parts for the queries, k_parts for the keys, as many for the values: the queries are bound by memory, keys
// and values by arithmetic, and beside each other they overlap (one workgroup for all three, one after the other, took a fifth more).  Medians: 32768
// tokens of 32 + 8 heads of 128 in bf16 172 us for 0.71 GB, 4.1 TB/s; 16 tokens 7.2 us, latencies.  Of these the certainty of codes takes 14 us (two
// conversions of each number, heads in 64 bits) and 1.5.
template <int DT, int LP, int PAIRS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    using T = typename Float<DT>::type;
    constexpr int SLOTS = 256 / LP;
    const int parts_of = a.q_parts + 2 * a.k_parts;
    const int group = hq::div_magic31(blockIdx.x, parts_of, a.part_magic.m, a.part_magic.s);
    const hq::Kv4Group g = group_of(a.c, group);
    if (g.count == 0) return;
    // slots: tokens, a power of two of them, times heads at once
    const int log2 = g.count > 4 ? 3 : g.count > 2 ? 2 : g.count - 1, at_once = SLOTS >> log2;
    const int in = kv4_block(threadIdx.x % LP), slot = threadIdx.x / LP, token = slot & ((1 << log2) - 1), first = slot >> log2;
    const bool live = in * 8 < a.c.d, mine = token < g.count;
    const int row = g.row + (mine ? token : 0);
    const int64_t place = g.s < a.c.batch ? g.position + (mine ? token : 0) : -1;
    int part = blockIdx.x - group * parts_of;
    if (part < a.q_parts)
        return turned_heads<T, LP, PAIRS, false>(a, part * at_once + first, a.q_parts * at_once, a.heads, row, place, in, live, mine, g);
    part -= a.q_parts;
    if (part < a.k_parts)
        return turned_heads<T, LP, PAIRS, true>(a, part * at_once + first, a.k_parts * at_once, a.c.kv_heads, row, place, in, live, mine, g);
    stored_heads<T, LP>(a, part - a.k_parts, log2, at_once, slot, first, row, place, in, live, mine, g);
}

// ---- read -------------------------------------------------------------------------------------------------------------
struct ReadArgs {
    hq::Kv4 c;
    void *k, *v;   // [t, kv_heads, d], dense
    int parts_log2;
};

// Workgroups of a group, side by side: the first half reads keys, the other values.  A slot has a row; of v it reads the dwords of its
// channels, which hold 8 tokens (the other slots that want them find them in the first-level cache).  Bound by what it writes: 131072 tokens of 8
// heads of 128 in bf16 147 us (median; 125 at best) for 0.68 GB, 4.6 TB/s.
template <int DT, int LP>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
    using T = typename Float<DT>::type;
    constexpr int SLOTS = 256 / LP;
    const hq::Kv4Group g = group_of(a.c, blockIdx.x >> a.parts_log2);
    if (g.count == 0) return;
    const int log2 = g.count > 4 ? 3 : g.count > 2 ? 2 : g.count - 1, at_once = SLOTS >> log2;
    const int in = kv4_block(threadIdx.x % LP), slot = threadIdx.x / LP, token = slot & ((1 << log2) - 1), first = slot >> log2;
    if (token >= g.count) return;   // (whole heads: no lane waits for another head's)
    const bool live = in * 8 < a.c.d;
    const int row = g.row + token, place = g.s < a.c.batch ? g.position + token : -1;
    const int64_t page = page_of(a.c, g);
    const float factor = walsh_factor(in, a.c.block_log2);
    const int parts = 1 << (a.parts_log2 - 1), part = blockIdx.x & (parts - 1), step = parts * at_once;
    const bool values = blockIdx.x & parts;
    T *const out = static_cast<T *>(values ? a.v : a.k) + static_cast<int64_t>(row) * a.c.kv_heads * a.c.d + in * 8;
    if (page < 0) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = place < 0 ? 0.0f : __builtin_nanf("");
        for (int h = part * at_once + first; h < a.c.kv_heads; h += step)
            if (live) store8(out + h * a.c.d, x);
        return;
    }
    const int64_t at = a.c.slots(page, 0) + a.c.slot(place), by_head = int64_t{1} << a.c.page_log2;
    const float *const scales = (values ? a.c.v_scale : a.c.k_scale) + at;
    const uint8_t *const codes = values ? a.c.v + (a.c.slots(page, 0) + a.c.slot(place & ~7)) * a.c.row_bytes() + (live ? in * 32 : 0)
                                        : a.c.k + at * a.c.row_bytes() + (live ? in * 4 : 0);
    const int shift = 4 * (place & 7);
    typedef uint32_t words4 __attribute__((ext_vector_type(4)));
    words4 raw[kAtOnce][2] = {};
    float raw_scale[kAtOnce] = {};
    const auto load = [&](int h) {
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e)
            if (h + e * step < a.c.kv_heads) {
                const uint8_t *p = codes + (h + e * step) * (by_head * a.c.row_bytes());
                raw_scale[e] = scales[(h + e * step) * by_head];
                if (values) {
                    raw[e][0] = reinterpret_cast<const words4 *>(p)[0];
                    raw[e][1] = reinterpret_cast<const words4 *>(p)[1];
                } else {
                    raw[e][0][0] = *reinterpret_cast<const uint32_t *>(p);
                }
            }
    };
    const auto work = [&](const words4 (&now)[2], float scale, int h) {
        const float f = scale * factor;
        uint32_t w = now[0][0];
        if (values) {
            w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w = __builtin_amdgcn_alignbit(now[i >> 2][i & 3] >> shift, w, 4);   // (its low 4 bits on top)
        }
        float x[8];
        kv4_floats(live ? w : 0u, x);
        walsh(x, in, a.c.block_log2);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= f;
        if (live) store8(out + h * a.c.d, x);
    };
    const int from = part * at_once + first;
    load(from);
    for (int h = from; h < a.c.kv_heads; h += kAtOnce * step) {
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e)
            if (h + e * step < a.c.kv_heads) work(raw[e], raw_scale[e], h + e * step);
        load(h + kAtOnce * step);
    }
}

// Workgroups that share a group's heads where there are few groups: one for each turn of 8 tokens, or of one where tokens come singly.
int parts_for(const hq::Kv4 &c, int groups, int heads, int lanes, int wanted) {
    const int slots = 256 / lanes, at_once = c.each == 1 && !c.begins ? slots : slots / 8;
    const int turns = (heads + at_once - 1) / at_once, more = (wanted * hq::compute_units() + groups - 1) / groups;
    return std::max(1, std::min({more, turns, 32}));
}

template <class F>
void with_lanes(int d, F f) {
    if (d <= 32) f(std::integral_constant<int, 4>{});
    else if (d <= 64) f(std::integral_constant<int, 8>{});
    else if (d <= 128) f(std::integral_constant<int, 16>{});
    else f(std::integral_constant<int, 32>{});
}
template <int DT>
void launch_append(AppendArgs a, hipStream_t st) {
    const int groups = hq::kv4_groups(a.c.t, a.c.batch), half = a.rotary >> 1;
    const Pairs pairs = a.interleaved || !a.rotary ? kNeighbours : half <= 64 && half >= 8 && hq::is_pow2(half) ? kLanes : half % 4 == 0 ? kQuads : kSingle;
    with_lanes(a.c.d, [&](auto lp) {
        constexpr int LP = decltype(lp)::value;
        a.q_parts = parts_for(a.c, groups, a.heads, LP, 8);
        a.k_parts = parts_for(a.c, groups, a.c.kv_heads, LP, 8);
        const unsigned parts = a.q_parts + 2 * a.k_parts, grid = static_cast<unsigned>(groups) * parts;
        a.part_magic = hq::magic31(parts);
        switch (pairs) {
            case kNeighbours: append_kernel<DT, LP, kNeighbours><<<grid, 256, 0, st>>>(a); break;
            case kLanes: append_kernel<DT, LP, kLanes><<<grid, 256, 0, st>>>(a); break;
            case kQuads: append_kernel<DT, LP, kQuads><<<grid, 256, 0, st>>>(a); break;
            default: append_kernel<DT, LP, kSingle><<<grid, 256, 0, st>>>(a); break;
        }
    });
}
template <int DT>
void launch_read(ReadArgs a, hipStream_t st) {
    const int groups = hq::kv4_groups(a.c.t, a.c.batch);
    with_lanes(a.c.d, [&](auto lp) {
        constexpr int LP = decltype(lp)::value;
        // (2366 tokens of 16 heads of 80: 16 workgroups a group 13 us, one for each turn of 8 tokens 7.6)
        const int parts = parts_for(a.c, groups, a.c.kv_heads, LP, 3);
        a.parts_log2 = 1;
        while (2 << (a.parts_log2 - 1) <= parts) ++a.parts_log2;
        read_kernel<DT, LP><<<static_cast<unsigned>(groups) << a.parts_log2, 256, 0, st>>>(a);
    });
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
                       norm != 0, eps, hq::magic31(c.d), {}, 0, 0};
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
    const ReadArgs a{c, k, v, 0};
    const hq::LaunchCheck check;
    const auto st = static_cast<hipStream_t>(stream);
    switch (dtype) {
        case HQ_F16: launch_read<HQ_F16>(a, st); break;
        case HQ_BF16: launch_read<HQ_BF16>(a, st); break;
        default: launch_read<HQ_F32>(a, st); break;
    }
    return check.status();
}
