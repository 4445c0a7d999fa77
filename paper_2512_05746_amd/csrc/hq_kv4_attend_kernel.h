// Attention over a 4-bit cache.  For a key head of one sequence, the rows are its new tokens times the query heads that share it:
//
//     s_rj = scale q_r k_j = scale (H q_r) . (codes of k_j) x k_scale_j,   o_r = H sum_j p_rj v_scale_j (codes of v_j) / sum_j p_rj
//
// with p the exponential of s minus a reference that follows the largest s so far: one pass over the cache.
//
// A wave holds tiles of 16 rows and takes 32 tokens a turn, all in registers: 4-bit codes turn into halves by one instruction for two,
// exactly, so that they go from memory to the matrix instruction without LDS.  Products are taken the other way round,
// S^T = K Q^T and O^T = V^T P^T: then a lane has one row of the tile throughout (its reference, its sum, its factor need no exchange), and the
// weights that leave the first product are in the lanes and in the order in which the second one takes them, if row m of the first tile of
// 16 tokens is token 8 (m / 4) + m % 4 and of the second 4 further on.  v is kept channel by channel for 8 tokens, the order of its operand.
//
// Roundings: H q to half (2^-11 of an element), in units of a power of two that leaves the row's largest below 2^12; weights times v_scale to
// half, in units of the power of two next to the largest v_scale so far (2^-11; below 2^-14 of it, 2^-25 of it).  With WIDE (32-bit
// results) both are two halves, 2^-22.  Codes are exact, sums are 32 bits.
//
// The reference moves only where s would exceed it by 8 (2^8 times 2 is far inside a half), so most turns leave the sums alone.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_floats.h"
#include "hq_kv4_attend.h"
#include "hq_kv4_lanes.h"

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) v += __shfl_xor(static_cast<long long>(v), i);
    return v;
}
__device__ __forceinline__ int wave_prefix(int v, int lane) {   // with its own
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
        const int o = __shfl_up(v, i);
        v += lane >= i ? o : 0;
    }
    return v;
}
// What the wave's lanes wrote to LDS, to be read by each other.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// Tokens of a part.
__device__ __forceinline__ int part_of(const hq::Kv4Attend &a, int lane) {
    if (!a.split) return hq::kKv4Undivided;
    int64_t work = 0;
    for (int base = 0; base < a.c.batch; base += 64)
        if (base + lane < a.c.batch) {
            const hq::Kv4Span p = hq::kv4_span(a.c, a.cut, base + lane);
            work += int64_t{p.blocks} * p.tokens;
        }
    return hq::kv4_part(a.cut, wave_sum(work), a.c.kv_heads);
}

// What a workgroup works on: a part of the tokens of a block of rows of one key head.
struct Task {
    int s, head, block, part, parts, slot;   // slot: its place among the parts' sums; s = -1: none, and `block` counts up from 0
};
__device__ __forceinline__ Task task_of(const hq::Kv4Attend &a, int id, int lane) {
    const int part = part_of(a, lane);
    int base = 0, slots = 0;
    for (int from = 0; from < a.c.batch; from += 64) {
        hq::Kv4Span p{};
        int parts = 1;
        if (from + lane < a.c.batch) {
            p = hq::kv4_span(a.c, a.cut, from + lane);
            parts = hq::kv4_parts(p, part);
        }
        const int count = p.blocks * parts * a.c.kv_heads, mine = parts > 1 ? count : 0;
        const int to = wave_prefix(count, lane), slot_to = wave_prefix(mine, lane);
        const uint64_t behind = __ballot(base + to > id);
        if (behind) {
            const int at = __ffsll(static_cast<unsigned long long>(behind)) - 1;
            const int in = id - base - __shfl(to - count, at), blocks = __shfl(p.blocks, at);
            parts = __shfl(parts, at);
            Task t;
            t.s = from + at;
            t.slot = slots + __shfl(slot_to - mine, at) + in;
            t.parts = parts;
            t.part = in % parts;
            t.block = in / parts % blocks;
            t.head = in / parts / blocks;
            return t;
        }
        base += __shfl(to, 63);
        slots += __shfl(slot_to, 63);
    }
    return {-1, 0, id - base, 0, 1, 0};
}

template <class F>
__device__ __forceinline__ void with_type(hq_dtype dt, F f) {
    if (dt == HQ_F16) f(static_cast<_Float16 *>(nullptr));
    else if (dt == HQ_BF16) f(static_cast<__bf16 *>(nullptr));
    else f(static_cast<float *>(nullptr));
}

// A row's result: its sums back through the transform, 8 channels a lane.
template <int KS>
__device__ __forceinline__ void store_row(const hq::Kv4Attend &a, float (&o)[8], float weight, int in, int64_t at) {
    const bool live = in * 8 < a.c.d;
    const float f = weight == 0.0f ? 0.0f : walsh_factor(a.c.block_log2) / weight;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = live && weight != 0.0f ? o[i] * f : 0.0f;
    walsh(o, in, a.c.block_log2);
    if (live) with_type(a.dtype, [&](auto *t) { store8(static_cast<decltype(t)>(a.out) + at + in * 8, o); });
}
template <int KS>
__device__ __forceinline__ void store_all(const hq::Kv4Attend &a, float value, int in, int64_t at) {
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = value;
    if (in * 8 < a.c.d) with_type(a.dtype, [&](auto *t) { store8(static_cast<decltype(t)>(a.out) + at + in * 8, o); });
}

constexpr int lanes_of(int ks) { return ks <= 1 ? 4 : ks <= 2 ? 8 : ks <= 4 ? 16 : 32; }   // that own a row, 8 channels each

// 32 tokens as they are in memory.
template <int KS> struct Turn32 {
    uint32_t k[2][KS], v[2 * KS];
    float4v ks[2], vs[2];
    bool bad;   // its group of tokens has no page
};
template <int N>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t *w) {
    typedef uint32_t words __attribute__((ext_vector_type(N == 3 ? 3 : N >= 4 ? 4 : N), aligned(4)));
    constexpr int STEP = N >= 4 ? 4 : N;
    const words t = *reinterpret_cast<const words *>(p);
#pragma unroll
    for (int i = 0; i < STEP; ++i) {
        if constexpr (N == 1) w[i] = __builtin_bit_cast(uint32_t, t);
        else w[i] = t[i];
    }
    if constexpr (N > STEP) load_words<N - STEP>(p + 4 * STEP, w + STEP);
}

template <int KS, int R, bool APART, bool WIDE>
__global__ __launch_bounds__(256) void attend_kernel(hq::Kv4Attend a) {
    constexpr int DP = 32 * KS, LP = lanes_of(KS), STAGE = DP + 8, ROW = DP + 4;
    // per wave: a tile of rows as halves (two planes where WIDE), and later their sums
    constexpr int WAVE_BYTES = 16 * ROW * 4 > 16 * STAGE * 2 * (1 + WIDE) ? 16 * ROW * 4 : 16 * STAGE * 2 * (1 + WIDE);
    __shared__ __attribute__((aligned(16))) uint8_t lds[4][WAVE_BYTES];
    __shared__ float row_factor[4][16], row_top[4][16], row_sum[4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const Task task = task_of(a, blockIdx.x, lane);
    const int in = lane % LP;
    if (task.s < 0) {
        // rows of no sequence: zeros
        const int begin = a.c.begin(a.c.batch), rows = (a.c.t - begin) * a.heads, from = blockIdx.x - task.block;
        const int step = (gridDim.x - from) * (256 / LP);
        for (int r = task.block * (256 / LP) + threadIdx.x / LP; r < rows; r += step)
            store_all<KS>(a, 0.0f, in, (begin + r / a.heads) * a.out_token + r % a.heads * a.out_head);
        return;
    }
    const int s = __builtin_amdgcn_readfirstlane(task.s), head = __builtin_amdgcn_readfirstlane(task.head);
    const hq::Kv4Span span = hq::kv4_span(a.c, a.cut, s);
    if (head >= a.c.kv_heads || (task.parts > 1 && task.slot >= a.slots)) return;
    const int group = a.cut.group, rows = span.n * group;   // (below 2^31: the host checks t x heads)
    const int row0 = task.block * a.cut.rows + (APART ? 0 : wave * 16 * R);
    const auto at_of = [&](int row, int64_t by_token, int64_t by_head) {
        return (span.begin + row / group) * by_token + (head * group + row % group) * by_head;
    };
    if (span.length > a.c.capacity()) {   // the sequence says that it has tokens that no page holds
        if (task.part == 0)
            for (int r = APART ? wave * (64 / LP) + lane / LP : lane / LP; r < 16 * R && row0 + r < rows; r += (APART ? 256 : 64) / LP)
                store_all<KS>(a, __builtin_nanf(""), in, at_of(row0 + r, a.out_token, a.out_head));
        return;
    }
    // ---- the rows: through the transform, to halves, to the lanes of the matrix instruction
    half8v q[R][KS], q_low[R][WIDE ? KS : 1];
    float factor[R];
    int position[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (APART && r) __syncthreads();
        uint8_t *const stage = lds[APART ? 0 : wave];
        for (int i = APART ? threadIdx.x / LP : lane / LP; i < 16; i += (APART ? 256 : 64) / LP) {
            const int row = row0 + 16 * r + i;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.0f;
            if (row < rows && in * 8 < a.c.d)
                with_type(a.dtype, [&](auto *t) { load8(static_cast<decltype(t)>(const_cast<void *>(a.q)) + at_of(row, a.q_token, a.q_head) + in * 8, x); });
            walsh(x, in, a.c.block_log2);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
            top = max_lanes<LP>(top);
            // x = x' 2^power, |x'| < 2^12: halves of full precision down to 2^-26 of the largest
            const int power = top == 0 || top >= 0x7F800000u ? 0 : __builtin_amdgcn_frexp_expf(__uint_as_float(top)) - 12;
            float f = __builtin_ldexpf(a.scale, power);
            const float sign = a.scale == 0.0f ? 0.0f : a.negative ? -1.0f : 1.0f;
            if (a.scale == 0.0f) f = 1.0f;
            if (top >= 0x7F800000u) f = __builtin_nanf("");
            half8v hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = top >= 0x7F800000u ? 0.0f : __builtin_ldexpf(x[e], -power) * sign;
                hi[e] = static_cast<_Float16>(y);
                lo[e] = static_cast<_Float16>(y - static_cast<float>(hi[e]));
            }
            if (in * 8 < DP) {
                *reinterpret_cast<half8v *>(stage + (i * STAGE + in * 8) * 2) = hi;
                if constexpr (WIDE) *reinterpret_cast<half8v *>(stage + (16 * STAGE + i * STAGE + in * 8) * 2) = lo;
            }
            if (in == 0) row_factor[APART ? 0 : wave][i] = f;
        }
        if constexpr (APART) __syncthreads();
        else wave_sync();
#pragma unroll
        for (int e = 0; e < KS; ++e) {
            q[r][e] = *reinterpret_cast<const half8v *>(stage + (m * STAGE + g * (DP / 4) + e * 8) * 2);
            if constexpr (WIDE) q_low[r][e] = *reinterpret_cast<const half8v *>(stage + (16 * STAGE + m * STAGE + g * (DP / 4) + e * 8) * 2);
        }
        factor[r] = row_factor[APART ? 0 : wave][m];
        const int row = row0 + 16 * r + m;
        position[r] = row < rows ? span.length - span.n + row / group : -1;
        if constexpr (!APART) wave_sync();
    }
    // ---- the tokens
    const int last_row = hq::kv4_min(row0 + 16 * R, rows) - 1;
    const int first_position = span.length - span.n + row0 / group, last_position = row0 < rows ? span.length - span.n + last_row / group : -1;
    const hq::Kv4Tiles tiles = hq::kv4_tiles(first_position, last_position, a.cut.window, a.cut.sinks);
    const int seen_from = hq::kv4_seen(last_position, a.cut.window, a.cut.sinks).from;
    const int share = ((tiles.count() + task.parts - 1) / task.parts + (APART ? 3 : 0)) & (APART ? ~3 : ~0);
    const int end = hq::kv4_min(tiles.count(), (task.part + 1) * share);
    int i = task.part * share + (APART ? wave : 0);
    constexpr int STEP = APART ? 4 : 1;

    const auto page_of = [&](int tile, int part) { return a.c.page(s, tile * 32 + 8 * part); };
    const auto load = [&](Turn32<KS> &t, int tile, int64_t k_page, int64_t v_page) {
        const int k_slot = a.c.slot(tile * 32 + 8 * (m >> 2)) + (m & 3), v_slot = a.c.slot(tile * 32 + 8 * g);
        t.bad = v_page < 0;
        const int64_t k_at = a.c.slots(k_page < 0 ? 0 : k_page, head), v_at = a.c.slots(v_page < 0 ? 0 : v_page, head) + v_slot;
        const uint8_t *k = a.c.k + (k_at + k_slot) * (DP / 2) + g * (KS * 4);
        load_words<KS>(k, t.k[0]);
        load_words<KS>(k + 4 * (DP / 2), t.k[1]);
        load_words<2 * KS>(a.c.v + v_at * (DP / 2) + m * (KS * 8), t.v);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            t.ks[e] = *reinterpret_cast<const float4v *>(a.c.k_scale + v_at + 4 * e);
            t.vs[e] = *reinterpret_cast<const float4v *>(a.c.v_scale + v_at + 4 * e);
        }
    };

    float4v o[R][2 * KS];
    float top[R], sum[R];            // the reference, this lane's sum of weights
    float limit = 0.0f, power = -100.0f;   // the largest v_scale that the reference allows for, its power of two
#pragma unroll
    for (int r = 0; r < R; ++r) {
        top[r] = -__builtin_inff();
        sum[r] = 0.0f;
#pragma unroll
        for (int e = 0; e < 2 * KS; ++e) o[r][e] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    Turn32<KS> next;
    int64_t k_page = -1, v_page = -1;
    if (i < end) {
        const int tile = tiles.tile(i);
        load(next, tile, page_of(tile, m >> 2), page_of(tile, g));
        if (i + STEP < end) {
            k_page = page_of(tiles.tile(i + STEP), m >> 2);
            v_page = page_of(tiles.tile(i + STEP), g);
        }
    }
    for (; i < end; i += STEP) {
        const int tile = tiles.tile(i);
        Turn32<KS> now = next;
        if (i + STEP < end) {
            load(next, tiles.tile(i + STEP), k_page, v_page);
            if (i + 2 * STEP < end) {
                k_page = page_of(tiles.tile(i + 2 * STEP), m >> 2);
                v_page = page_of(tiles.tile(i + 2 * STEP), g);
            }
        }
        float4v t[R][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int r = 0; r < R; ++r) t[r][h] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < KS; ++e) {
                const half8v k = kv4_halves(now.k[h][e]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if constexpr (WIDE) t[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q_low[r][e], t[r][h], 0, 0, 0);
                    t[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[r][e], t[r][h], 0, 0, 0);
                }
            }
        }
        if (now.bad) now.ks[0] = now.ks[1] = float4v{1.0f, 1.0f, 1.0f, 1.0f} * __builtin_nanf("");
        const int first = tile * 32;
        const bool whole = first + 31 <= first_position && (first >= seen_from || first + 32 <= a.cut.sinks);
        const int token = first + 8 * g;
        if (!whole) {
            // scales behind the sequence's end are whatever the page held
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (token + 4 * h + e >= span.length) now.ks[h][e] = now.vs[h][e] = 0.0f;
        }
        uint32_t seen[R];   // a bit for each of the lane's 8 tokens
        float most[R];
        bool move = false;
        float v_top = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) v_top = fmaxf(v_top, now.vs[h][e]);
        move = v_top >= limit;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            seen[r] = 0xFFu;
            if (!whole) {
                const int from = a.cut.window > 0 && position[r] >= a.cut.window ? position[r] - a.cut.window + 1 : 0;
                seen[r] = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = token + e;
                    if (j <= position[r] && (j >= from || j < a.cut.sinks)) seen[r] |= 1u << e;
                }
            }
            most[r] = -__builtin_inff();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                t[r][h] *= now.ks[h];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!whole && !(seen[r] >> (4 * h + e) & 1)) t[r][h][e] = -__builtin_inff();
                    most[r] = fmaxf(most[r], t[r][h][e]);
                }
            }
            most[r] *= factor[r];
            move |= most[r] > top[r] - power + 8.0f;
        }
        if (__any(move)) {
            v_top = fmaxf(v_top, __shfl_xor(v_top, 16));
            v_top = fmaxf(v_top, __shfl_xor(v_top, 32));
            const float before = power;
            if (v_top >= limit && v_top > 0.0f) {
                const int p = hq::kv4_max(-100, hq::kv4_min(100, __builtin_amdgcn_frexp_expf(v_top) - 1));
                power = fmaxf(power, static_cast<float>(p));
                limit = __builtin_ldexpf(2.0f, static_cast<int>(power));
                if (power == 100.0f) limit = __builtin_inff();
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top_here = fmaxf(most[r], __shfl_xor(most[r], 16));
                top_here = fmaxf(top_here, __shfl_xor(top_here, 32));
                const float moved = fmaxf(top[r] - before, top_here) + power;
                const float by = top[r] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top[r] - moved);
                top[r] = moved;
                sum[r] *= by;
#pragma unroll
                for (int e = 0; e < 2 * KS; ++e) o[r][e] *= by;
            }
        }
        half8v p[R], p_low[WIDE ? R : 1];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float reference = top[r] == -__builtin_inff() ? 0.0f : top[r];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = __builtin_amdgcn_exp2f(fmaf(t[r][h][e], factor[r], -reference));
                    float y = w * now.vs[h][e];
                    if (!whole && !(seen[r] >> (4 * h + e) & 1)) w = y = 0.0f;
                    sum[r] += w;
                    p[r][4 * h + e] = static_cast<_Float16>(y);
                    if constexpr (WIDE) p_low[r][4 * h + e] = static_cast<_Float16>(y - static_cast<float>(p[r][4 * h + e]));
                }
        }
#pragma unroll
        for (int e = 0; e < 2 * KS; ++e) {
            const half8v v = kv4_halves(now.v[e]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (WIDE) o[r][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p_low[r], o[r][e], 0, 0, 0);
                o[r][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[r], o[r][e], 0, 0, 0);
            }
        }
    }
    // ---- the waves' sums together, and out
#pragma unroll
    for (int r = 0; r < R; ++r) {
        sum[r] += __shfl_xor(sum[r], 16);
        sum[r] += __shfl_xor(sum[r], 32);
        if constexpr (APART) __syncthreads();
        else wave_sync();
        float *const mine = reinterpret_cast<float *>(lds[wave]);
        // lane (m, g) has channels 2 KS (4 g + i) + e of row m
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < 2 * KS; c += 2) {
                typedef float float2v __attribute__((ext_vector_type(2)));
                *reinterpret_cast<float2v *>(mine + m * ROW + 2 * KS * (4 * g + e) + c) = float2v{o[r][c][e], o[r][c + 1][e]};
            }
        if (g == 0) {
            row_top[wave][m] = top[r];
            row_sum[wave][m] = sum[r];
        }
        if constexpr (APART) __syncthreads();
        else wave_sync();
        for (int i2 = APART ? threadIdx.x / LP : lane / LP; i2 < 16; i2 += (APART ? 256 : 64) / LP) {
            const int row = row0 + 16 * r + i2;
            if (row >= rows) continue;
            float x[8], weight, reference;
            if constexpr (APART) {
                reference = fmaxf(fmaxf(row_top[0][i2], row_top[1][i2]), fmaxf(row_top[2][i2], row_top[3][i2]));
                weight = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float by = row_top[w][i2] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(row_top[w][i2] - reference);
                    weight += by * row_sum[w][i2];
                    if (in * 8 < DP) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] += by * reinterpret_cast<const float *>(lds[w])[i2 * ROW + in * 8 + e];
                    }
                }
            } else {
                reference = row_top[wave][i2];
                weight = row_sum[wave][i2];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = in * 8 < DP ? mine[i2 * ROW + in * 8 + e] : 0.0f;
            }
            if (task.parts == 1) {
                store_row<KS>(a, x, weight, in, at_of(row, a.out_token, a.out_head));
            } else {
                const int64_t at = int64_t{task.slot} * a.cut.rows + (APART ? 0 : wave * 16 * R) + 16 * r + i2;
                if (in * 8 < DP) store8(a.sums + at * DP + in * 8, x);
                if (in == 0) {
                    a.tops[2 * at] = reference;
                    a.tops[2 * at + 1] = weight;
                }
            }
        }
    }
}

// The parts of a row's tokens together: a workgroup for each row of a call whose tokens may be apart.
template <int KS>
__global__ __launch_bounds__(256) void join_kernel(hq::Kv4Attend a) {
    constexpr int DP = 32 * KS, LP = lanes_of(KS), SLOTS = 256 / LP;
    __shared__ float x_of[SLOTS][LP * 8 + 4], top_of[SLOTS], sum_of[SLOTS];
    const int lane = threadIdx.x & 63, token = blockIdx.x / a.heads, q_head = blockIdx.x % a.heads;
    const int part = part_of(a, lane);
    int s = -1, slots = 0;
    for (int from = 0; from <= a.c.batch; from += 64) {
        const int at = from + lane;
        const bool before = at <= a.c.batch && a.c.begin(at) <= token;
        s += __popcll(__ballot(before));
    }
    if (s >= a.c.batch) return;
    // (of sequences without tokens the last one that begins here)
    for (int from = 0; from < s; from += 64) {
        int mine = 0;
        if (from + lane < s) {
            const hq::Kv4Span p = hq::kv4_span(a.c, a.cut, from + lane);
            const int parts = hq::kv4_parts(p, part);
            mine = parts > 1 ? p.blocks * parts * a.c.kv_heads : 0;
        }
        slots += static_cast<int>(wave_sum(mine));
    }
    const hq::Kv4Span span = hq::kv4_span(a.c, a.cut, s);
    const int parts = hq::kv4_parts(span, part);
    if (parts == 1 || span.length > a.c.capacity()) return;
    const int group = a.cut.group, row = (token - span.begin) * group + q_head % group, block = row / a.cut.rows;
    const int64_t before = int64_t{slots} + (int64_t{q_head / group} * span.blocks + block) * parts;
    if (before < 0 || before + parts > a.slots) return;
    const int64_t first = before * a.cut.rows + row % a.cut.rows;
    const int in = threadIdx.x % LP, slot = threadIdx.x / LP;
    float x[8], top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    const auto add = [&](float other_top, float other_sum, const float (&other)[8]) {
        if (other_sum == 0.0f) return;   // (a row that is NaN has no reference, but a sum)
        const float to = fmaxf(top, other_top);
        const float mine = top == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top - to), by = __builtin_amdgcn_exp2f(other_top - to);
        top = to;
        sum = sum * mine + other_sum * by;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * mine + other[e] * by;
    };
    for (int p = slot; p < parts; p += SLOTS) {
        const int64_t at = first + int64_t{p} * a.cut.rows;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.0f;
        if (in * 8 < DP) load8(a.sums + at * DP + in * 8, y);
        add(a.tops[2 * at], a.tops[2 * at + 1], y);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x_of[slot][in * 8 + e] = x[e];
    if (in == 0) {
        top_of[slot] = top;
        sum_of[slot] = sum;
    }
    __syncthreads();
    if (slot) return;
    for (int p = 1; p < SLOTS && p < parts; ++p) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x_of[p][in * 8 + e];
        add(top_of[p], sum_of[p], y);
    }
    store_row<KS>(a, x, sum, in, token * a.out_token + q_head * a.out_head);
}

}  // namespace

namespace hq {

template <int KS>
void kv4_attend_launch(const Kv4Attend &a, Kv4Shape shape, unsigned blocks, hipStream_t st) {
    const auto go = [&](auto tiles, auto apart, auto wide) {
        attend_kernel<KS, decltype(tiles)::value, decltype(apart)::value, decltype(wide)::value><<<blocks, 256, 0, st>>>(a);
    };
    const auto with_wide = [&](auto tiles, auto apart) {
        if (a.dtype == HQ_F32) go(tiles, apart, std::true_type{});
        else go(tiles, apart, std::false_type{});
    };
    if (shape.apart && shape.tiles == 1) with_wide(std::integral_constant<int, 1>{}, std::true_type{});
    else if (shape.tiles == 1) with_wide(std::integral_constant<int, 1>{}, std::false_type{});
    else if constexpr (KS <= 4) {
        if (shape.apart) with_wide(std::integral_constant<int, 2>{}, std::true_type{});
        else with_wide(std::integral_constant<int, 2>{}, std::false_type{});
    }
    if (a.split) join_kernel<KS><<<static_cast<unsigned>(a.c.t) * a.heads, 256, 0, st>>>(a);
}

}  // namespace hq
