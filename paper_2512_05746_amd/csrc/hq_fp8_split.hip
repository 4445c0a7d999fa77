// Product of E4M3 codes for few tokens or few tiles: the waves of a workgroup share one small tile of results and split K.
//
// A wave takes every NW-th step of 128 codes: weights and activations go from memory straight into its registers (a row's 128 bytes
// of a step are read whole, by 4 lanes), there is no barrier before the end, where the waves' sums meet in LDS, in the order of the waves.
// Activations come as codes with their scales, or as 16- or 32-bit floats, which the wave then quantises itself (a lane holds 32
// neighbours of a token's 128: the maximum is one over 4 lanes), so that a whole layer is one launch; each workgroup of the same tokens
// quantises them anew.
//
// Bound by latency (launch, one round of loads for each step of a wave, the exchange), for many channels and few tokens by reading the weights: us in
// a graph, bf16: a layer of 960 -> 3840 for 1 token 3.4 (on codes 2.6), for 64 tokens 4.9 (3.5); 16 tokens of 4096 -> 4096 8.9 (6.2: 33 MB with
// the codes of the tokens, 16.8 of them from memory); 1 token of 4096 -> 8192 9.6 (8.8: 33.5 MB, the launch aside at the rate of a large copy).  The tile kernel
// takes 4.8, 5.1, 11.9 and 11.9 us on codes.  Loads of two or four steps at once changed nothing.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "hq_common.h"
#include "hq_fp8.h"
#include "hq_fp8_codes.h"
#include "hq_fp8_product.h"

namespace {

constexpr int kCodes = -1;   // input type: codes
constexpr int NW = 8;        // waves of a workgroup

struct SplitArgs {
    ProductArgs p;
    const void *x;        // activations that are quantised here
    int64_t row_stride;
    int k;
};

// tile (bx, by) of channels and tokens; part: [NW][16 MT][16 NT + 4]
template <int IN, int OUT, int MT, int NT>
__device__ __forceinline__ void split(const SplitArgs &a, uint32_t bx, uint32_t by, float *part) {
    using Out = typename Float<OUT>::type;
    constexpr bool kFp32 = OUT == HQ_F32;
    constexpr int TM = MT * 16, TN = NT * 16, PITCH = TN + 4;   // floats of a token's row in LDS
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t m0 = static_cast<int64_t>(by) * TM;
    const int n0 = bx * TN;
    const int rows_x = a.p.m - m0 < TM ? static_cast<int>(a.p.m - m0) : TM, rows_w = a.p.n - n0 < TN ? a.p.n - n0 : TN;
    const uint32_t pitch = a.p.pitch;
    const __amdgpu_buffer_rsrc_t wb = buffer_of(a.p.w + static_cast<int64_t>(n0) * pitch, static_cast<uint32_t>(rows_w) * pitch);
    const __amdgpu_buffer_rsrc_t xb = buffer_of(IN == kCodes ? a.p.x + m0 * pitch : a.p.w, static_cast<uint32_t>(rows_x) * pitch);
    const float *sw = a.p.sw + static_cast<int64_t>(n0 / kStep) * a.p.sw_block;

    int x_row[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) x_row[j] = j * 16 + l16 < rows_x ? j * 16 + l16 : rows_x - 1;
    f32x4 acc[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int step = wave; step < a.p.steps; step += NW) {
        const uint32_t c = step * kStep + quarter * 32;
        // (pieces beyond a row's end: zeros from beyond the buffer.)  Row r of tile i holds channel 4 NT (r / 4) + 4 i + r % 4, which makes a
        // lane's channels neighbours.
        const uint32_t lo_at = c < pitch ? c : 0x80000000u, hi_at = c + 16 < pitch ? c + 16 : 0x80000000u;
        v8i w[NT], x[MT];
        float s[MT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const uint32_t row = static_cast<uint32_t>((l16 >> 2) * (4 * NT) + i * 4 + (l16 & 3)) * pitch;
            w[i] = __builtin_shufflevector(buffer_load16(wb, row + lo_at, 0), buffer_load16(wb, row + hi_at, 0), 0, 1, 2, 3, 4, 5, 6, 7);
        }
        const float s_w = sw[static_cast<int64_t>(step) * a.p.sw_step];
        if constexpr (IN == kCodes) {
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const uint32_t row = static_cast<uint32_t>(x_row[j]) * pitch;
                x[j] = __builtin_shufflevector(buffer_load16(xb, row + lo_at, 0), buffer_load16(xb, row + hi_at, 0), 0, 1, 2, 3, 4, 5, 6, 7);
                s[j] = a.p.sx[static_cast<int64_t>(step) * a.p.m + m0 + x_row[j]];
            }
        } else {
            using T = typename Float<IN == kCodes ? HQ_F32 : IN>::type;
            Raw8<T> raw[MT][4];
            const bool whole = (step + 1) * kStep <= a.k;   // (of all lanes)
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const T *from = static_cast<const T *>(a.x) + (m0 + x_row[j]) * a.row_stride + c;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int left = a.k - static_cast<int>(c) - q * 8;
                    if (whole || left >= 8) raw[j][q].load(from + q * 8);
                    else if (left > 0) raw[j][q].load_some(from + q * 8, left);
                    else raw[j][q].zero();
                }
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                Tops<T> tops;
#pragma unroll
                for (int q = 0; q < 4; ++q) tops.add(raw[j][q]);
                uint32_t top = tops.all();
                top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16)));
                top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
                s[j] = scale_of(top);
                const float inverse = inverse_of(s[j]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[8];
                    raw[j][q].floats(v);
                    x[j][2 * q] = static_cast<int>(codes4(v, inverse));
                    x[j][2 * q + 1] = static_cast<int>(codes4(v + 4, inverse));
                }
            }
        }
        Halves xh[kFp32 ? MT : 1];
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            if constexpr (kFp32) xh[j] = halves_of(x[j]);
            s[j] *= s_w;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            f32x4 p[MT];
            if constexpr (!kFp32) {
#pragma unroll
                for (int j = 0; j < MT; ++j) p[j] = mfma_fp8(w[i], x[j]);
            } else {
                const Halves wh = halves_of(w[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < MT; ++j)
                        p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wh.v[k], xh[j].v[k], k ? p[j] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[j][e], s[j], acc[i][j][e]);
        }
    }

    // the waves' sums
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < NT; ++i)
            *reinterpret_cast<f32x4 *>(part + (wave * TM + j * 16 + l16) * PITCH + quarter * 4 * NT + i * 4) = acc[i][j];
    __syncthreads();
    for (int e = tid; e < TM * TN / 4; e += NW * 64) {
        const int row = e / (TN / 4), c = e % (TN / 4) * 4;
        if (row >= rows_x || c >= rows_w) continue;
        f32x4 sum = *reinterpret_cast<const f32x4 *>(part + row * PITCH + c);
        for (int w = 1; w < NW; ++w) sum += *reinterpret_cast<const f32x4 *>(part + (w * TM + row) * PITCH + c);
        Out *y = static_cast<Out *>(a.p.y) + (m0 + row) * a.p.n + n0 + c;
        const Out *bias = static_cast<const Out *>(a.p.bias) + n0 + c;
        if (c + 4 <= rows_w) {
            typename Vec<Out, 4>::type v, b;
            if (a.p.bias) b = load_vec<Out, 4>(bias);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = round_to<Out>(a.p.bias ? sum[i] + static_cast<float>(b[i]) : sum[i]);
            store_vec<Out, 4>(y, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < rows_w) y[i] = round_to<Out>(a.p.bias ? sum[i] + static_cast<float>(bias[i]) : sum[i]);
        }
    }
}

template <int IN, int OUT, int MT, int NT>
__global__ __launch_bounds__(NW * 64) void split_kernel(SplitArgs a) {
    extern __shared__ __attribute__((aligned(16))) float part[];
    split<IN, OUT, MT, NT>(a, blockIdx.x, blockIdx.y, part);
}

// Two products of codes, `b` with fp32 results, and sums: workgroups of b first, then of a, then of the sums.
template <int OUT, int MT, int NT>
__global__ __launch_bounds__(NW * 64) void pair_kernel(SplitArgs a, SplitArgs b, hq::Fp8Sums sums, uint32_t a_across, uint32_t b_across, uint32_t a_groups,
                                                       uint32_t b_groups) {
    extern __shared__ __attribute__((aligned(16))) float part[];
    if (blockIdx.x < b_groups) {
        split<kCodes, HQ_F32, MT, NT>(b, blockIdx.x % b_across, blockIdx.x / b_across, part);
    } else if (blockIdx.x < b_groups + a_groups) {
        const uint32_t i = blockIdx.x - b_groups;
        split<kCodes, OUT, MT, NT>(a, i % a_across, i / a_across, part);
    } else {
        sum_rows(sums, blockIdx.x - b_groups - a_groups, threadIdx.x, part);
    }
}

constexpr int lds_bytes(int mt, int nt) { return NW * mt * 16 * (nt * 16 + 4) * 4; }

template <int IN, int OUT, int MT, int NT>
hq_status launch(const SplitArgs &a, hipStream_t st) {
    constexpr auto kernel = split_kernel<IN, OUT, MT, NT>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    const dim3 grid((a.p.n + NT * 16 - 1) / (NT * 16), static_cast<uint32_t>((a.p.m + MT * 16 - 1) / (MT * 16)));
    const hq::LaunchCheck check;
    kernel<<<grid, NW * 64, lds_bytes(MT, NT), st>>>(a);
    return check.status();
}

template <int OUT, int MT, int NT>
hq_status launch_pair(const SplitArgs &a, const SplitArgs &b, const hq::Fp8Sums &sums, hipStream_t st) {
    constexpr auto kernel = pair_kernel<OUT, MT, NT>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    const auto across = [](const SplitArgs &x) { return static_cast<uint32_t>((x.p.n + NT * 16 - 1) / (NT * 16)); };
    const auto groups = [&](const SplitArgs &x) { return across(x) * static_cast<uint32_t>((x.p.m + MT * 16 - 1) / (MT * 16)); };
    const uint32_t ga = groups(a), gb = groups(b);
    const hq::LaunchCheck check;
    kernel<<<ga + gb + sum_blocks(sums), NW * 64, lds_bytes(MT, NT), st>>>(a, b, sums, across(a), across(b), ga, gb);
    return check.status();
}
template <int OUT>
hq_status pair_with_cut(const SplitArgs &a, const SplitArgs &b, const hq::Fp8Sums &sums, hq::Fp8Cut cut, hipStream_t st) {
    if (cut.mt == 1 && cut.nt == 1) return launch_pair<OUT, 1, 1>(a, b, sums, st);
    if (cut.mt == 1 && cut.nt == 2) return launch_pair<OUT, 1, 2>(a, b, sums, st);
    return launch_pair<OUT, 2, 2>(a, b, sums, st);
}

template <int IN, int OUT>
hq_status with_cut(const SplitArgs &a, hq::Fp8Cut cut, hipStream_t st) {
    if (cut.mt == 1 && cut.nt == 1) return launch<IN, OUT, 1, 1>(a, st);
    if (cut.mt == 1 && cut.nt == 2) return launch<IN, OUT, 1, 2>(a, st);
    if constexpr (IN == kCodes) return launch<IN, OUT, 2, 2>(a, st);
    else return launch<IN, OUT, 1, 4>(a, st);
}
template <int IN>
hq_status with_out(const SplitArgs &a, hq::Fp8Cut cut, hq_dtype out, hipStream_t st) {
    return out == HQ_F16 ? with_cut<IN, HQ_F16>(a, cut, st) : out == HQ_BF16 ? with_cut<IN, HQ_BF16>(a, cut, st) : with_cut<IN, HQ_F32>(a, cut, st);
}

}  // namespace

namespace hq {

namespace {
// One round of a wave takes `round` us (latency), a workgroup's share of one step `each` us of a CU that has several; measured with 1 x 960 -> 3840,
// 16 x 4096 -> 4096, 64 x 960 -> 3840 (rounds), 2048 x 3840 -> 960 and 960 x 4096 -> 256 (shares), us without the launch.  Activations of
// 32 bits are twice the loads, and quantising costs each workgroup: there a workgroup takes more channels (16 x 64) where on codes it takes more of
// both (32 x 32; 16 x 64 is slower by 0 .. 20 % there, 32 x 32 by 10 .. 20 % here).
struct Cost {
    int mt, nt;
    float round[3], each[3];   // codes; 16-bit, 32-bit activations

    int64_t groups(int64_t m, int64_t n) const { return ((m + 16 * mt - 1) / (16 * mt)) * ((n + 16 * nt - 1) / (16 * nt)); }
    float shares(int64_t m, int64_t n, int64_t steps, int kind, hq_dtype out) const {   // us, of all workgroups, of all CUs
        return static_cast<float>(groups(m, n)) * steps * each[kind] * (out == HQ_F32 && !kind ? 1.2f : 1.0f);
    }
    float rounds(int64_t steps, int kind) const { return round[kind] * ((steps + NW - 1) / NW); }
};
constexpr float kNot = 1e30f;
constexpr Cost costs[] = {{1, 1, {1.0f, 1.5f, 2.0f}, {0.113f, 0.165f, 0.33f}},
                          {1, 2, {1.4f, 1.6f, 2.3f}, {0.17f, 0.25f, 0.51f}},
                          {1, 4, {kNot, 2.6f, 3.0f}, {0.30f, 0.365f, 0.65f}},
                          {2, 2, {1.9f, kNot, kNot}, {0.245f, 0.373f, 1.1f}}};
constexpr float kBegin = 2.2f;
}  // namespace

Fp8Cut fp8_split_cut(int64_t m, int64_t n, int64_t steps, const hq_dtype *in, hq_dtype out) {
    const int kind = !in ? 0 : *in == HQ_F32 ? 2 : 1;
    const float cu = static_cast<float>(compute_units());
    Fp8Cut best{1, 1, 1e30f};
    for (const Cost &c : costs) {
        if ((m + 16 * c.mt - 1) / (16 * c.mt) > 65535) continue;   // (the grid's limit in y)
        // Fewer workgroups than CUs: each has a CU of its own.  Those that quantise keep a CU's vector units busy, so that a second one on it waits (333 x
        // 1024 -> 768 5.7 us, -> 777 8.6); those on codes wait for loads.
        float share = std::max(c.shares(m, n, steps, kind, out) / cu, c.shares(1, 1, steps, kind, out));
        if (in) share = ceilf(static_cast<float>(c.groups(m, n)) / cu) * c.shares(1, 1, steps, kind, out);
        const float us = kBegin + std::max(c.rounds(steps, kind), share);
        if (us < best.us) best = {c.mt, c.nt, us};
    }
    return best;
}

Fp8Cut fp8_split_pair_cut(const Fp8Product &a, const Fp8Product &b, hq_dtype out) {
    const float cu = static_cast<float>(compute_units());
    Fp8Cut best{1, 1, 1e30f};
    for (const Cost &c : costs) {
        if (c.groups(a.m, a.n) + c.groups(b.m, b.n) > 0x3FFFFFFF) continue;
        const float share = std::max((c.shares(a.m, a.n, a.steps, 0, out) + c.shares(b.m, b.n, b.steps, 0, HQ_F32)) / cu,
                                     c.shares(1, 1, std::max(a.steps, b.steps), 0, HQ_F32));
        const float us = kBegin + std::max(c.rounds(std::max(a.steps, b.steps), 0), share);
        if (us < best.us) best = {c.mt, c.nt, us};
    }
    return best;
}

hq_status fp8_split_pair(const Fp8Product &a, const Fp8Product &b, const Fp8Sums &sums, Fp8Cut cut, hq_dtype out, hipStream_t st) {
    const SplitArgs x{a, nullptr, 0, 0}, y{b, nullptr, 0, 0};
    return out == HQ_F16 ? pair_with_cut<HQ_F16>(x, y, sums, cut, st) : out == HQ_BF16 ? pair_with_cut<HQ_BF16>(x, y, sums, cut, st)
                                                                                      : pair_with_cut<HQ_F32>(x, y, sums, cut, st);
}

hq_status fp8_split(const Fp8Product &p, Fp8Cut cut, const void *x, hq_dtype x_dtype, int64_t row_stride, int k, hq_dtype out, hipStream_t st) {
    const SplitArgs a{p, x, row_stride, k};
    if (!x) return with_out<kCodes>(a, cut, out, st);
    switch (x_dtype) {
        case HQ_F16: return with_out<HQ_F16>(a, cut, out, st);
        case HQ_BF16: return with_out<HQ_BF16>(a, cut, out, st);
        default: return with_out<HQ_F32>(a, cut, out, st);
    }
}

}  // namespace hq
