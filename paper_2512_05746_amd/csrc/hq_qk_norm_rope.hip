// Norm of every query and key head and its rotation by the token's position, in one pass, and the gradients of that.
//
//     r = (mean x^2 + eps)^-1/2,   n = x r w,   y = R(position) n
//
// R turns the channel pairs (i, i + R/2), or (2i, 2i + 1), of the first R = rotary channels by the angles of the token's position; the
// other channels pass.  Backwards, with g = R^T dy (the opposite angles):
//
//     dw_i = sum over tokens and heads of g_i x_i r,     dx = r (g w - x r mean(g w x r))
//
// A token with a negative position is padding: zeros, and no part in the sums.  A position beyond the tables gives NaN.
//
// All sums in fp32; one rounding, of the result.
//
// Bound by memory (two passes over q and k, three backwards).  A head is owned by G neighbouring lanes, a lane owns C channel pairs: it
// loads C channels of each half of the head (or 2 C neighbours, where these are the pairs), so that both channels of a pair meet in one
// lane and only the sum of squares crosses lanes (permutes inside a row of 16).  Heads that no such cut fits (more than 64 lanes of the
// pairs that divide both their rotated and their other channels) take a wave each, whose lanes have pairs 64 apart.
// 65536 tokens of 32 + 8 heads of 128 in bf16: 252 us (5.3 TB/s, a large copy 5.15); backwards, 32768 tokens: 191 us and 4.5 for the
// weights' sums (5.2 TB/s).  Few tokens are bound by latency: launch, the position, the tables' row that it names, results (1 token 2.5
// us, 1021 tokens of 32 heads of 72 in fp16 5.7).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hq_common.h"
#include "hq_floats.h"
#include "hq_fp8.h"
#include "hq_qk_cut.h"

namespace {

struct Heads {              // q or k
    const void *x, *dy, *w;
    void *out;              // y, or dx
    float *dw;              // [channels]
    int64_t x_token, x_head, dy_token, dy_head, out_token, out_head;   // strides, in elements
    uint32_t heads, items;  // items: tokens x heads
    uint32_t magic, shift;  // exact division by heads
    uint32_t blocks;        // workgroups that work on these heads
};

struct QkArgs {
    Heads part[2];          // queries, keys
    const float *cos, *sin; // [positions, rotary / 2]
    const void *pos;        // int32 or int64 per token, or null: the token's index
    int pos_wide;
    int64_t positions;
    int d, rotary, interleaved, w_float;
    float eps;
    float *sums;            // [workgroups, d]: backwards, every workgroup's part of dw
};

// what a token's position asks for
struct Turn {
    bool pad, beyond;
    const float *cos, *sin;
};
__device__ __forceinline__ Turn turn_of(const QkArgs &a, uint32_t token) {
    int64_t p = token;
    if (a.pos) p = a.pos_wide ? static_cast<const int64_t *>(a.pos)[token] : static_cast<const int32_t *>(a.pos)[token];
    const bool pad = p < 0, beyond = p >= a.positions;
    const int64_t row = (pad || beyond ? 0 : p) * (a.rotary >> 1);
    return {pad, beyond, a.cos + row, a.sin + row};
}

template <class T, int N>
__device__ __forceinline__ void load_floats(const T *p, float *v) {
    constexpr int STEP = 16 / static_cast<int>(sizeof(T)) < N ? 16 / static_cast<int>(sizeof(T)) : N;
#pragma unroll
    for (int i = 0; i < N; i += STEP) {
        const typename Vec<T, STEP>::type t = load_vec<T, STEP>(p + i);
#pragma unroll
        for (int e = 0; e < STEP; ++e) v[i + e] = static_cast<float>(t[e]);
    }
}
template <class T, int N>
__device__ __forceinline__ void store_floats(T *p, const float *v) {
    constexpr int STEP = 16 / static_cast<int>(sizeof(T)) < N ? 16 / static_cast<int>(sizeof(T)) : N;
#pragma unroll
    for (int i = 0; i < N; i += STEP) {
        typename Vec<T, STEP>::type t;
#pragma unroll
        for (int e = 0; e < STEP; ++e) t[e] = round_to<T>(v[i + e]);
        store_vec<T, STEP>(p + i, t);
    }
}
template <class T, int N>
__device__ __forceinline__ void load_weights(const QkArgs &a, const void *w, int at, float *v) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = 1.0f;
    } else if (a.w_float) {
        load_floats<float, N>(static_cast<const float *>(w) + at, v);
    } else {
        load_floats<T, N>(static_cast<const T *>(w) + at, v);
    }
}

// (u, v) <- pairs turned by the angles; with -sin the other way round
template <int C>
__device__ __forceinline__ void rotate(bool interleaved, const float *c, const float *s, float sign, float *u, float *v) {
    if (interleaved) {
        // pairs are neighbours: pair i of the first half of the registers, then of the second
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float &x = 2 * i < C ? u[2 * i] : v[2 * i - C];
            float &y = 2 * i + 1 < C ? u[2 * i + 1] : v[2 * i + 1 - C];
            const float si = s[i] * sign, nx = x * c[i] - y * si, ny = y * c[i] + x * si;
            x = nx;
            y = ny;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const float si = s[i] * sign, nx = u[i] * c[i] - v[i] * si, ny = v[i] * c[i] + u[i] * si;
            u[i] = nx;
            v[i] = ny;
        }
    }
}

template <int DT, int C, int G, bool BACK>
__global__ __launch_bounds__(256) void heads_kernel(QkArgs a) {
    using T = typename Float<DT>::type;
    constexpr int SLOTS = 256 / G;
    const bool keys = blockIdx.x >= a.part[0].blocks;
    const Heads &h = a.part[keys];
    const uint32_t block = keys ? blockIdx.x - a.part[0].blocks : blockIdx.x;
    const int in = threadIdx.x % G, slot = threadIdx.x / G;
    const hq::QkLane lane = hq::qk_lane_of(a.d, a.rotary, a.interleaved, C, in);
    const bool live = lane.live;
    const int p = lane.p;
    const hq::QkPlace at = lane.at;
    float w1[C], w2[C];
    load_weights<T, C>(a, h.w, at.first, w1);
    load_weights<T, C>(a, h.w, at.second, w2);
    float dw1[C], dw2[C];
    if constexpr (BACK) {
#pragma unroll
        for (int i = 0; i < C; ++i) dw1[i] = dw2[i] = 0.0f;
    }
    const float inv_d = 1.0f / static_cast<float>(a.d);
    // (every lane of a wave goes through the same turns: an item beyond the last is worked on as the last, and dropped)
    for (uint32_t base = block * SLOTS; base < h.items; base += h.blocks * SLOTS) {
        const bool mine = base + slot < h.items;
        const uint32_t item = mine ? base + slot : h.items - 1;
        const uint32_t token = hq::div_magic31(item, h.heads, h.magic, h.shift), head = item - token * h.heads;
        const Turn t = turn_of(a, token);   // (first: the tables' addresses wait for it)
        const T *x = static_cast<const T *>(h.x) + static_cast<int64_t>(token) * h.x_token + static_cast<int64_t>(head) * h.x_head;
        float u[C], v[C], gu[C], gv[C], c[C], s[C];
        load_floats<T, C>(x + at.first, u);
        load_floats<T, C>(x + at.second, v);
        if constexpr (BACK) {
            const T *dy = static_cast<const T *>(h.dy) + static_cast<int64_t>(token) * h.dy_token + static_cast<int64_t>(head) * h.dy_head;
            load_floats<T, C>(dy + at.first, gu);
            load_floats<T, C>(dy + at.second, gv);
        }
        if (at.rotated) {
            load_floats<float, C>(t.cos + p, c);
            load_floats<float, C>(t.sin + p, s);
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < C; ++i) sum += u[i] * u[i] + v[i] * v[i];
        sum = sum_lanes<G>(live ? sum : 0.0f);
        float rstd = 1.0f / sqrtf(sum * inv_d + a.eps);
        if (t.beyond) rstd = __builtin_nanf("");
        T *out = static_cast<T *>(h.out) + static_cast<int64_t>(token) * h.out_token + static_cast<int64_t>(head) * h.out_head;
        if constexpr (!BACK) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                u[i] *= rstd * w1[i];
                v[i] *= rstd * w2[i];
            }
            if (at.rotated) rotate<C>(a.interleaved, c, s, 1.0f, u, v);
        } else {
            if (at.rotated) rotate<C>(a.interleaved, c, s, -1.0f, gu, gv);
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                u[i] *= rstd;   // the normalised values
                v[i] *= rstd;
                if (mine && !t.pad) {
                    dw1[i] += gu[i] * u[i];
                    dw2[i] += gv[i] * v[i];
                }
                gu[i] *= w1[i];
                gv[i] *= w2[i];
                dot += gu[i] * u[i] + gv[i] * v[i];
            }
            dot = sum_lanes<G>(live ? dot : 0.0f) * inv_d;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                u[i] = rstd * (gu[i] - u[i] * dot);
                v[i] = rstd * (gv[i] - v[i] * dot);
            }
        }
        if (t.pad) {
#pragma unroll
            for (int i = 0; i < C; ++i) u[i] = v[i] = 0.0f;
        }
        if (live && mine) {
            store_floats<T, C>(out + at.first, u);
            store_floats<T, C>(out + at.second, v);
        }
    }
    if constexpr (BACK) {
        // the workgroup's part of dw: slots summed in order through LDS
        extern __shared__ float part[];   // [SLOTS][2 C G]
#pragma unroll
        for (int i = 0; i < C; ++i) {
            part[slot * 2 * C * G + in * C + i] = dw1[i];
            part[slot * 2 * C * G + C * G + in * C + i] = dw2[i];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * C * G; e += 256) {
            float sum = 0.0f;
            for (int i = 0; i < SLOTS; ++i) sum += part[i * 2 * C * G + e];
            const bool other = e >= C * G;
            const hq::QkLane l = hq::qk_lane_of(a.d, a.rotary, a.interleaved, C, (other ? e - C * G : e) / C);
            const hq::QkPlace q = l.at;
            const int k = e % C;
            if (l.live) {
                a.sums[static_cast<int64_t>(blockIdx.x) * a.d + (other ? q.second : q.first) + k] = sum;
            }
        }
    }
}

// Any even number of channels up to 1024: a wave for each head, a lane's pairs 64 apart (4096 tokens of 16 + 1 heads in bf16: of 514
// channels, 258 of them turned, 96 us, of 1024, 66 turned, 154; 1024 all turned, which the kernel above takes, 56).
constexpr int kMostPairs = 8;   // of a lane
template <int DT, bool BACK>
__global__ __launch_bounds__(256) void wave_kernel(QkArgs a) {
    using T = typename Float<DT>::type;
    const bool keys = blockIdx.x >= a.part[0].blocks;
    const Heads &h = a.part[keys];
    const uint32_t block = keys ? blockIdx.x - a.part[0].blocks : blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.d >> 1;
    float dw1[kMostPairs], dw2[kMostPairs];
#pragma unroll
    for (int i = 0; i < kMostPairs; ++i) dw1[i] = dw2[i] = 0.0f;
    const float inv_d = 1.0f / static_cast<float>(a.d);
    for (uint32_t item = block * 4 + wave; item < h.items; item += h.blocks * 4) {
        const uint32_t token = hq::div_magic31(item, h.heads, h.magic, h.shift), head = item - token * h.heads;
        const T *x = static_cast<const T *>(h.x) + static_cast<int64_t>(token) * h.x_token + static_cast<int64_t>(head) * h.x_head;
        const T *dy = static_cast<const T *>(h.dy) + static_cast<int64_t>(token) * h.dy_token + static_cast<int64_t>(head) * h.dy_head;
        T *out = static_cast<T *>(h.out) + static_cast<int64_t>(token) * h.out_token + static_cast<int64_t>(head) * h.out_head;
        const Turn t = turn_of(a, token);
        float u[kMostPairs], v[kMostPairs], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kMostPairs; ++i) {
            u[i] = v[i] = 0.0f;
            const int p = lane + 64 * i;
            if (p < pairs) {
                const hq::QkPlace at = hq::qk_place_of(a.d, a.rotary, a.interleaved, 1, p);
                u[i] = static_cast<float>(x[at.first]);
                v[i] = static_cast<float>(x[at.second]);
            }
            sum += u[i] * u[i] + v[i] * v[i];
        }
        float rstd = 1.0f / sqrtf(sum_lanes<64>(sum) * inv_d + a.eps);
        if (t.beyond) rstd = __builtin_nanf("");
        float dot = 0.0f;
        float gu[kMostPairs], gv[kMostPairs];
#pragma unroll
        for (int i = 0; i < kMostPairs; ++i) {
            u[i] *= rstd;
            v[i] *= rstd;
            const int p = lane + 64 * i;
            if (BACK && p < pairs) {
                const hq::QkPlace at = hq::qk_place_of(a.d, a.rotary, a.interleaved, 1, p);
                float gx = static_cast<float>(dy[at.first]), gy = static_cast<float>(dy[at.second]), w1, w2;
                if (at.rotated) rotate<1>(false, t.cos + p, t.sin + p, -1.0f, &gx, &gy);
                load_weights<T, 1>(a, h.w, at.first, &w1);
                load_weights<T, 1>(a, h.w, at.second, &w2);
                if (!t.pad) {
                    dw1[i] += gx * u[i];
                    dw2[i] += gy * v[i];
                }
                gu[i] = gx * w1;
                gv[i] = gy * w2;
                dot += gu[i] * u[i] + gv[i] * v[i];
            }
        }
        if (BACK) dot = sum_lanes<64>(dot) * inv_d;
#pragma unroll
        for (int i = 0; i < kMostPairs; ++i) {
            const int p = lane + 64 * i;
            if (p >= pairs) continue;
            const hq::QkPlace at = hq::qk_place_of(a.d, a.rotary, a.interleaved, 1, p);
            float y1, y2;
            if constexpr (BACK) {
                y1 = rstd * (gu[i] - u[i] * dot);
                y2 = rstd * (gv[i] - v[i] * dot);
            } else {
                float w1, w2;
                load_weights<T, 1>(a, h.w, at.first, &w1);
                load_weights<T, 1>(a, h.w, at.second, &w2);
                y1 = u[i] * w1;
                y2 = v[i] * w2;
                if (at.rotated) rotate<1>(false, t.cos + p, t.sin + p, 1.0f, &y1, &y2);
            }
            out[at.first] = round_to<T>(t.pad ? 0.0f : y1);
            out[at.second] = round_to<T>(t.pad ? 0.0f : y2);
        }
    }
    if constexpr (BACK) {
        __shared__ float part[4][1024];
#pragma unroll
        for (int i = 0; i < kMostPairs; ++i) {
            const int p = lane + 64 * i;
            if (p < pairs) {
                const hq::QkPlace at = hq::qk_place_of(a.d, a.rotary, a.interleaved, 1, p);
                part[wave][at.first] = dw1[i];
                part[wave][at.second] = dw2[i];
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.d; e += 256)
            a.sums[static_cast<int64_t>(blockIdx.x) * a.d + e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
    }
}

// dw of queries (workgroups of the first half) and keys: the workgroups' parts, of which there are up to 1024.  8 channels a workgroup,
// 128 threads to a channel with 8 loads under way each: one round of them, where the parts come from other XCDs' caches (1024 parts of
// 128 channels: 22 us with 16 threads and one load after the other, 13 with 32 and 4 loads).
__global__ __launch_bounds__(1024) void weight_sums_kernel(QkArgs a) {
    __shared__ float s[128][8];
    const uint32_t half = gridDim.x >> 1;
    const bool keys = blockIdx.x >= half;
    const Heads &h = a.part[keys];
    const int x = threadIdx.x & 7, y = threadIdx.x >> 3, c = (blockIdx.x - (keys ? half : 0)) * 8 + x;
    const float *sums = a.sums + (keys ? static_cast<int64_t>(a.part[0].blocks) * a.d : 0) + c;
    float sum = 0.0f;
    if (c < a.d)
        for (uint32_t r = y; r < h.blocks; r += 1024) {
            float t[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const uint32_t row = r + 128 * i;
                const float v = sums[static_cast<int64_t>(row < h.blocks ? row : r) * a.d];
                t[i] = row < h.blocks ? v : 0.0f;
            }
            sum += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
    s[y][x] = sum;
    __syncthreads();
    if (y < 16) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += s[y + 16 * i][x];
    }
    __syncthreads();
    if (y < 16) s[y][x] = sum;
    __syncthreads();
    if (y == 0 && c < a.d && h.dw) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += s[i][x];
        h.dw[c] = sum;
    }
}

// Forwards 24 workgroups a CU (65536 tokens of 40 heads of 128 in 16 bits: 252 us, 290 with a workgroup for every 32 heads, 259 with 8 a
// CU); backwards, where a workgroup keeps sums, 4 (2 to 8 within 1 %).
uint32_t blocks_for(uint32_t items, int slots, bool back) {
    const uint32_t all = (items + slots - 1) / slots;
    return std::min<uint32_t>(all, static_cast<uint32_t>(hq::compute_units()) * (back ? 4 : 24));
}

template <int DT, bool BACK>
void launch(const QkArgs &a, hq::QkCut cut, hipStream_t st) {
    const uint32_t blocks = a.part[0].blocks + a.part[1].blocks;
    if (blocks) {
        const auto go = [&](auto c, auto g) {
            constexpr int C = decltype(c)::value, G = decltype(g)::value;
            heads_kernel<DT, C, G, BACK><<<blocks, 256, BACK ? 256 * 2 * C * 4 : 0, st>>>(a);
        };
        const auto with_c = [&](auto c) {
            switch (cut.g) {
                case 2: return go(c, std::integral_constant<int, 2>{});
                case 4: return go(c, std::integral_constant<int, 4>{});
                case 8: return go(c, std::integral_constant<int, 8>{});
                case 16: return go(c, std::integral_constant<int, 16>{});
                case 32: return go(c, std::integral_constant<int, 32>{});
                default: return go(c, std::integral_constant<int, 64>{});
            }
        };
        if (cut.c == 8) with_c(std::integral_constant<int, 8>{});
        else if (cut.c == 4) with_c(std::integral_constant<int, 4>{});
        else if (cut.c == 2) with_c(std::integral_constant<int, 2>{});
        else if (cut.c == 1) with_c(std::integral_constant<int, 1>{});
        else wave_kernel<DT, BACK><<<blocks, 256, 0, st>>>(a);
    }
    if (BACK) weight_sums_kernel<<<2 * ((a.d + 7) / 8), 1024, 0, st>>>(a);
}

template <bool BACK>
hq_status run(const QkArgs &a, hq_dtype dt, hq::QkCut cut, hipStream_t st) {
    const hq::LaunchCheck check;
    switch (dt) {
        case HQ_F16: launch<HQ_F16, BACK>(a, cut, st); break;
        case HQ_BF16: launch<HQ_BF16, BACK>(a, cut, st); break;
        default: launch<HQ_F32, BACK>(a, cut, st); break;
    }
    return check.status();
}

hq_status check_sizes(int64_t t, int heads, int kv_heads, int d, int rotary, int64_t positions, const void *pos, int pos_size, float eps) {
    if (t < 0 || heads <= 0 || kv_heads <= 0 || d <= 0 || rotary < 0 || rotary > d || positions <= 0) return HQ_ERR_SHAPE;
    if ((d & 1) || (rotary & 1) || (!pos && t > positions)) return HQ_ERR_SHAPE;
    if (!(eps >= 0.0f)) return HQ_ERR_SHAPE;
    if (pos && pos_size != 4 && pos_size != 8) return HQ_ERR_DTYPE;
    if (d > 1024 || t > 0x7FFF0000 || t * std::max(heads, kv_heads) > 0x7FFF0000) return HQ_ERR_UNSUPPORTED;
    return HQ_OK;
}

void fill(Heads &h, int64_t t, int heads, int slots, bool back) {
    h.heads = heads;
    h.items = static_cast<uint32_t>(t * heads);
    const hq::Magic31 m = hq::magic31(heads);
    h.magic = m.m;
    h.shift = m.s;
    h.blocks = blocks_for(h.items, slots, back);
}

}  // namespace

extern "C" hq_status hq_qk_norm_rope(const void *q, const void *k, hq_dtype dtype, int64_t t, int heads, int kv_heads, int d,
                                     const int64_t *strides, const void *q_weight, const void *k_weight, hq_dtype w_dtype,
                                     const float *cos, const float *sin, int64_t positions, int rotary, int interleaved, const void *pos,
                                     int pos_size, float eps, void *q_out, void *k_out, void *stream) {
    if ((t > 0 && (!q || !k || !q_out || !k_out)) || !strides || (rotary > 0 && (!cos || !sin))) return HQ_ERR_NULL;
    if (!hq::is_float(dtype) || (w_dtype != dtype && w_dtype != HQ_F32)) return HQ_ERR_DTYPE;
    if (const hq_status s = check_sizes(t, heads, kv_heads, d, rotary, positions, pos, pos_size, eps)) return s;
    const int size = hq::size_of(dtype);
    for (const void *p : {q, k, static_cast<const void *>(q_out), static_cast<const void *>(k_out)})
        if (!hq::aligned_to(p, size)) return HQ_ERR_ALIGN;
    for (const void *p : {q_weight, k_weight})
        if (!hq::aligned_to(p, hq::size_of(w_dtype))) return HQ_ERR_ALIGN;
    if (!hq::aligned_to(cos, 4) || !hq::aligned_to(sin, 4) || !hq::aligned_to(pos, pos_size == 8 ? 8 : 4)) return HQ_ERR_ALIGN;
    const hq::QkCut cut = hq::qk_cut_of(d, rotary, dtype, false);
    const int slots = cut.g ? 256 / cut.g : 4;
    QkArgs a{};
    a.part[0] = Heads{q, nullptr, q_weight, q_out, nullptr, strides[0], strides[1], 0, 0, strides[4], strides[5]};
    a.part[1] = Heads{k, nullptr, k_weight, k_out, nullptr, strides[2], strides[3], 0, 0, strides[6], strides[7]};
    fill(a.part[0], t, heads, slots, false);
    fill(a.part[1], t, kv_heads, slots, false);
    a.cos = cos, a.sin = sin, a.pos = pos, a.pos_wide = pos_size == 8, a.positions = positions;
    a.d = d, a.rotary = rotary, a.interleaved = interleaved != 0, a.w_float = w_dtype == HQ_F32, a.eps = eps;
    return run<false>(a, dtype, cut, static_cast<hipStream_t>(stream));
}

extern "C" int64_t hq_qk_norm_rope_backward_workspace(hq_dtype dtype, int64_t t, int heads, int kv_heads, int d, int rotary) {
    if (!hq::is_float(dtype) || check_sizes(t, heads, kv_heads, d, rotary, 1, &t, 4, 0.0f) != HQ_OK) return 0;
    const hq::QkCut cut = hq::qk_cut_of(d, rotary, dtype, true);
    const int slots = cut.g ? 256 / cut.g : 4;
    const int64_t blocks = int64_t{blocks_for(static_cast<uint32_t>(t * heads), slots, true)} +
                           blocks_for(static_cast<uint32_t>(t * kv_heads), slots, true);
    return blocks * d * 4;
}

extern "C" hq_status hq_qk_norm_rope_backward(const void *dq, const void *dk, const void *q, const void *k, hq_dtype dtype, int64_t t,
                                              int heads, int kv_heads, int d, const int64_t *strides, const void *q_weight,
                                              const void *k_weight, hq_dtype w_dtype, const float *cos, const float *sin,
                                              int64_t positions, int rotary, int interleaved, const void *pos, int pos_size,
                                              float eps, void *workspace, void *q_grad, void *k_grad, float *q_weight_grad,
                                              float *k_weight_grad, void *stream) {
    if ((t > 0 && (!dq || !dk || !q || !k || !q_grad || !k_grad)) || !strides || (rotary > 0 && (!cos || !sin))) return HQ_ERR_NULL;
    if (!hq::is_float(dtype) || (w_dtype != dtype && w_dtype != HQ_F32)) return HQ_ERR_DTYPE;
    if (const hq_status s = check_sizes(t, heads, kv_heads, d, rotary, positions, pos, pos_size, eps)) return s;
    if (t > 0 && !workspace) return HQ_ERR_NULL;   // (sizes that are refused have a workspace of no bytes)
    const int size = hq::size_of(dtype);
    for (const void *p : {dq, dk, q, k, static_cast<const void *>(q_grad), static_cast<const void *>(k_grad)})
        if (!hq::aligned_to(p, size)) return HQ_ERR_ALIGN;
    for (const void *p : {q_weight, k_weight})
        if (!hq::aligned_to(p, hq::size_of(w_dtype))) return HQ_ERR_ALIGN;
    if (!hq::aligned_to(cos, 4) || !hq::aligned_to(sin, 4) || !hq::aligned_to(pos, pos_size == 8 ? 8 : 4) ||
        !hq::aligned_to(workspace, 4) || !hq::aligned_to(q_weight_grad, 4) || !hq::aligned_to(k_weight_grad, 4))
        return HQ_ERR_ALIGN;
    const hq::QkCut cut = hq::qk_cut_of(d, rotary, dtype, true);
    const int slots = cut.g ? 256 / cut.g : 4;
    QkArgs a{};
    a.part[0] = Heads{q, dq, q_weight, q_grad, q_weight_grad, strides[0], strides[1], strides[4], strides[5], strides[8], strides[9]};
    a.part[1] = Heads{k, dk, k_weight, k_grad, k_weight_grad, strides[2], strides[3], strides[6], strides[7], strides[10], strides[11]};
    fill(a.part[0], t, heads, slots, true);
    fill(a.part[1], t, kv_heads, slots, true);
    a.cos = cos, a.sin = sin, a.pos = pos, a.pos_wide = pos_size == 8, a.positions = positions;
    a.d = d, a.rotary = rotary, a.interleaved = interleaved != 0, a.w_float = w_dtype == HQ_F32, a.eps = eps;
    a.sums = static_cast<float *>(workspace);
    return run<true>(a, dtype, cut, static_cast<hipStream_t>(stream));
}
