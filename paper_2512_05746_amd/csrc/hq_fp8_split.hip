// Product of E4M3 codes for few tokens or few tiles: the waves of a workgroup share one small tile of results and split K.
//
// A wave takes every NW-th step of 128 codes.  They go from memory into LDS that the wave has to itself, from there into its registers,
// and while it multiplies them the next ones are on their way; there is no barrier before the end, where the waves' sums meet in LDS, in
// the order of the waves.  Activations come as codes with their scales, or as 16- or 32-bit floats, which the wave then quantises itself
// (16 lanes to a token, 8 neighbours to a lane), so that a whole layer is one launch; each workgroup of the same tokens quantises them
// anew.
//
// Why LDS, where every byte is read once: a matrix instruction wants neighbouring lanes to hold neighbouring rows, and loads for which
// they are take the path to memory 64 cycles each (16 bytes a cycle and CU), loads whose neighbouring lanes read 128 neighbouring bytes a
// quarter of that.  Straight into registers 64 tokens of 4096 -> 4096 took 10.1 us on codes, 512 of 4096 -> 512 9.7, 16 of 4096 -> 8192
// 7.9; so 6.3, 5.6 and 5.3.
//
// Bound by latency (launch, one round of loads for each step of a wave, the exchange), for many channels and few tokens by reading the
// weights: us in a graph, bf16 on codes: 960 -> 3840 for 1 token 2.6, for 64 3.3; 16 tokens of 4096 -> 4096 4.3, 1 token of 4096 -> 8192
// 4.6 (tiles: 4.8, 5.1, 11.9 and 11.9).  As a layer in one launch, fp16: 3.2, 4.7, 8.4 and 6.3.  (The estimates below charge that form
// for 16 tokens whatever their count, so one token of 4096 -> 8192 takes two launches: 7.0 in a graph, 7.3 called one by one.)
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
constexpr int NW = 8;        // most waves of a workgroup

struct SplitArgs {
    ProductArgs p;
    const void *x;        // activations that are quantised here
    int64_t row_stride;
    int k;
};

// bytes of LDS of a wave: the codes of a step, [token or channel][8 pieces of 16 bytes], in the end its sums, [16 MT][16 NT + 4]
constexpr int wave_bytes(int mt, int nt) { return std::max((mt + nt) * 16 * kStep, mt * 16 * (nt * 16 + 4) * 4); }

// tile (bx, by) of channels and tokens
template <int IN, int OUT, int MT, int NT>
__device__ __forceinline__ void split(const SplitArgs &a, uint32_t bx, uint32_t by, uint8_t *lds) {
    using Out = typename Float<OUT>::type;
    using T = typename Float<IN == kCodes ? HQ_F32 : IN>::type;
    constexpr bool kFp32 = OUT == HQ_F32;
    constexpr int TM = MT * 16, TN = NT * 16, PITCH = TN + 4, AREA = wave_bytes(MT, NT);   // pitch: floats of a token's sums in LDS
    static_assert(IN == kCodes || MT == 1, "values of 16 tokens");
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = static_cast<int>(blockDim.x >> 6);
    const int64_t m0 = static_cast<int64_t>(by) * TM;
    const int n0 = bx * TN;
    const int rows_x = a.p.m - m0 < TM ? static_cast<int>(a.p.m - m0) : TM, rows_w = a.p.n - n0 < TN ? a.p.n - n0 : TN;
    const uint32_t pitch = a.p.pitch;
    const v4i wb = words_of(a.p.w + static_cast<int64_t>(n0) * pitch, static_cast<uint32_t>(rows_w) * pitch);
    const v4i xb = words_of(IN == kCodes ? a.p.x + m0 * pitch : a.p.w, static_cast<uint32_t>(rows_x) * pitch);
    const float *sw = a.p.sw + static_cast<int64_t>(n0 / kStep) * a.p.sw_block;
    uint8_t *const mine = lds + wave * AREA;
    const uint32_t mine_at = lds_address(lds) + wave * AREA;

    // A load brings 8 rows, lane = (row, piece): the lanes of a row read 128 neighbouring bytes.  Row r of tile i holds channel
    // 4 NT (r / 4) + 4 i + r % 4, which makes a lane's channels neighbours; pieces are in an order that depends on the row (key), so that
    // reads of a column of rows use all banks.  Rows beyond the last, and pieces beyond a row's end, are zeros from beyond the buffer.
    const int r8 = lane >> 3;
    const uint32_t piece = ((lane & 7) ^ (r8 >> 1)) * 16, x_off = static_cast<uint32_t>(r8) * pitch,
                   w_off = static_cast<uint32_t>((r8 >> 2) * (4 * NT) + (r8 & 3)) * pitch;
    const auto request = [&](int step) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t c = static_cast<uint32_t>(step) * kStep + (piece ^ h * 64), beyond = c < pitch ? 0 : 0x80000000u;
            if constexpr (IN == kCodes) {
#pragma unroll
                for (int j = 0; j < MT; ++j)
                    load16_to_lds(xb, beyond ? beyond : x_off + static_cast<uint32_t>(j * 16 + h * 8) * pitch + c,
                                  mine_at + (j * 2 + h) * 1024);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i)
                load16_to_lds(wb, beyond ? beyond : w_off + static_cast<uint32_t>(i * 4 + h * 8 * NT) * pitch + c,
                              mine_at + MT * 2048 + (i * 2 + h) * 1024);
        }
    };
    // values of row 4 i + lane / 16, 8 neighbours to a lane
    Raw8<T> raw[4];
    const auto request_values = [&](int step) {
        const int c = step * kStep + l16 * 8, left = a.k - c;
        const bool whole = (step + 1) * kStep <= a.k;   // (of all lanes)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i * 4 < rows_x) {
                const int row = i * 4 + quarter < rows_x ? i * 4 + quarter : rows_x - 1;
                const T *from = static_cast<const T *>(a.x) + (m0 + row) * a.row_stride + c;
                if (whole || left >= 8) raw[i].load(from);
                else if (left > 0) raw[i].load_some(from, left);
                else raw[i].zero();
            }
        }
    };
    float s[MT], s_w = 0.0f;   // scales of the step that is under way
    const auto request_scales = [&](int step) {
        s_w = sw[static_cast<int64_t>(step) * a.p.sw_step];
        if constexpr (IN == kCodes) {
#pragma unroll
            for (int j = 0; j < MT; ++j)
                s[j] = a.p.sx[static_cast<int64_t>(step) * a.p.m + m0 + (j * 16 + l16 < rows_x ? j * 16 + l16 : rows_x - 1)];
        }
    };
    // the lane's two pieces of row l16 of a tile
    const uint32_t at0 = l16 * kStep + ((quarter * 2) ^ (l16 >> 1)) * 16, at1 = at0 ^ 16;
    const auto fetch = [&](int tile) {
        return __builtin_shufflevector(*reinterpret_cast<const v4i *>(mine + tile * 2048 + at0),
                                       *reinterpret_cast<const v4i *>(mine + tile * 2048 + at1), 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f32x4 acc[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < MT; ++j) s[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i].zero();

    if (wave < a.p.steps) {
        request_scales(wave);
        request(wave);
        if constexpr (IN != kCodes) request_values(wave);
    }
    for (int step = wave; step < a.p.steps; step += NW) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // (the scales are here: what is requested below is not waited for on their account)
        asm volatile("" : "+v"(s_w));
        float scale[MT];
        if constexpr (IN == kCodes) {
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                asm volatile("" : "+v"(s[j]));
                scale[j] = s[j] * s_w;
            }
        } else {
            // (beyond the last row what LDS holds goes into results that are not stored)
            uint32_t top = 0;   // of row l16 % 4, of the lane's four
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i * 4 < rows_x) {
                    Tops<T> tops;
                    tops.add(raw[i]);
                    const uint32_t t = max_lanes<16>(tops.all());
                    top = (l16 & 3) == i ? t : top;
                }
            }
            const float its_scale = scale_of(top);
            const int its_inverse = __float_as_int(inverse_of(its_scale));
            // of the quad's lanes 0 .. 3
            const float inverse[4] = {__int_as_float(dpp<0x00>(its_inverse)), __int_as_float(dpp<0x55>(its_inverse)),
                                      __int_as_float(dpp<0xAA>(its_inverse)), __int_as_float(dpp<0xFF>(its_inverse))};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i * 4 < rows_x) {
                    float v[8];
                    raw[i].floats(v);
                    const int row = i * 4 + quarter;
                    *reinterpret_cast<v2i *>(mine + row * kStep + ((l16 >> 1) ^ (row >> 1)) * 16 + (l16 & 1) * 8) =
                        v2i{static_cast<int>(codes4(v, inverse[i])), static_cast<int>(codes4(v + 4, inverse[i]))};
                }
            }
            // to the lanes of the tokens: row l16 is part l16 / 4 of lanes 16 (l16 % 4) ..
            scale[0] = __shfl(its_scale, (l16 & 3) * 16 + (l16 >> 2)) * s_w;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (codes of other lanes are read)
        }
        v8i w[NT], x[MT];
#pragma unroll
        for (int j = 0; j < MT; ++j) x[j] = fetch(j);
#pragma unroll
        for (int i = 0; i < NT; ++i) w[i] = fetch(MT + i);
        if (step + NW < a.p.steps) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (read before it is filled again)
            request_scales(step + NW);
            request(step + NW);
            if constexpr (IN != kCodes) request_values(step + NW);
        }
        Halves xh[kFp32 ? MT : 1];
        if constexpr (kFp32) {
#pragma unroll
            for (int j = 0; j < MT; ++j) xh[j] = halves_of(x[j]);
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
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[j][e], scale[j], acc[i][j][e]);
        }
    }

    // the waves' sums, each wave's where its codes were
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    float *const sums = reinterpret_cast<float *>(mine);
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < NT; ++i) *reinterpret_cast<f32x4 *>(sums + (j * 16 + l16) * PITCH + quarter * 4 * NT + i * 4) = acc[i][j];
    __syncthreads();
    const float *const part = reinterpret_cast<const float *>(lds);
    for (int e = tid; e < TM * TN / 4; e += waves * 64) {
        const int row = e / (TN / 4), c = e % (TN / 4) * 4;
        if (row >= rows_x || c >= rows_w) continue;
        f32x4 sum = *reinterpret_cast<const f32x4 *>(part + row * PITCH + c);
        const auto add = [&](int w) { sum += *reinterpret_cast<const f32x4 *>(part + w * (AREA / 4) + row * PITCH + c); };
        if (waves == NW) {
#pragma unroll
            for (int w = 1; w < NW; ++w) add(w);
        } else {
            for (int w = 1; w < waves; ++w) add(w);
        }
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
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    split<IN, OUT, MT, NT>(a, blockIdx.x, blockIdx.y, lds);
}

// Two products of codes, `b` with fp32 results, and sums: workgroups of b first, then of a, then of the sums.
template <int OUT, int MT, int NT>
__global__ __launch_bounds__(NW * 64) void pair_kernel(SplitArgs a, SplitArgs b, hq::Fp8Sums sums, uint32_t a_across, uint32_t b_across,
                                                       uint32_t a_groups, uint32_t b_groups) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    if (blockIdx.x < b_groups) {
        split<kCodes, HQ_F32, MT, NT>(b, blockIdx.x % b_across, blockIdx.x / b_across, lds);
    } else if (blockIdx.x < b_groups + a_groups) {
        const uint32_t i = blockIdx.x - b_groups;
        split<kCodes, OUT, MT, NT>(a, i % a_across, i / a_across, lds);
    } else {
        sum_rows(sums, blockIdx.x - b_groups - a_groups, threadIdx.x, reinterpret_cast<float *>(lds));
    }
}

// (a wave for each step, up to NW: those without a step would keep LDS from other workgroups)
int waves_of(int steps) { return std::min(NW, steps); }

template <int IN, int OUT, int MT, int NT>
hq_status launch(const SplitArgs &a, hipStream_t st) {
    constexpr auto kernel = split_kernel<IN, OUT, MT, NT>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    const dim3 grid((a.p.n + NT * 16 - 1) / (NT * 16), static_cast<uint32_t>((a.p.m + MT * 16 - 1) / (MT * 16)));
    const hq::LaunchCheck check;
    kernel<<<grid, waves_of(a.p.steps) * 64, waves_of(a.p.steps) * wave_bytes(MT, NT), st>>>(a);
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
    const int waves = std::max(4, waves_of(std::max(a.p.steps, b.p.steps)));   // (the sums take 4)
    const hq::LaunchCheck check;
    kernel<<<ga + gb + sum_blocks(sums), waves * 64, waves * wave_bytes(MT, NT), st>>>(a, b, sums, across(a), across(b), ga, gb);
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
    if constexpr (IN == kCodes) {
        if (cut.mt == 2) return launch<IN, OUT, 2, 2>(a, st);
        return launch<IN, OUT, 4, 4>(a, st);
    } else {
        if (cut.nt == 4) return launch<IN, OUT, 1, 4>(a, st);
        return launch<IN, OUT, 1, 8>(a, st);
    }
}
template <int IN>
hq_status with_out(const SplitArgs &a, hq::Fp8Cut cut, hq_dtype out, hipStream_t st) {
    return out == HQ_F16    ? with_cut<IN, HQ_F16>(a, cut, st)
           : out == HQ_BF16 ? with_cut<IN, HQ_BF16>(a, cut, st)
                            : with_cut<IN, HQ_F32>(a, cut, st);
}

}  // namespace

namespace hq {

namespace {
// A launch takes `begin` us, one round of a wave `round` (latency), a workgroup `fixed` and `each` for a step of a CU that has several;
// measured with 1 and 16 x 960 -> 3840, 16 and 64 x 4096 -> 4096 (rounds), 512 x 4096 -> 512 and 2048, 512 x 1024 -> 2048, 2048 x 2048 ->
// 2048 and 2048 x 512 -> 2048 (shares), us in a graph; fp32: what a workgroup takes longer with fp32 results.  On codes a cut of 64 x 64
// is for products that give every CU one of them (512 x 4096 -> 2048 10.3 us, 32 x 32 13.9, 64 x 64 tiles 13.0); between those 32 x 64 is
// no faster than the better of its neighbours by more than 6 %.  Activations that are quantised: there a workgroup takes more channels
// (16 x 64: 333 x 1024 -> 768 4.6 us, 16 x 32 5.4, 16 x 128 5.2; 16 x 128 where these are more than the CUs: 512 x 1024 -> 1024 5.5, 16 x
// 64 6.1, 32-bit 6.4 and 8.4).
struct Cost {
    int mt, nt;
    float begin, fp32, fixed[3], round[3], each[3];   // codes; 16-bit, 32-bit activations

    int64_t groups(int64_t m, int64_t n) const { return ((m + 16 * mt - 1) / (16 * mt)) * ((n + 16 * nt - 1) / (16 * nt)); }
    // (of two products the one with fewer steps has waves that only wait: 1.8 times the fixed part, 2048 x 512 -> 2048 with 8 waves 16.0
    // us, with 4 11.5)
    float workgroup(int64_t steps, int kind, hq_dtype out, bool pair = false) const {
        return (fixed[kind] * (pair ? 1.8f : 1.0f) + steps * each[kind]) * (out == HQ_F32 && !kind ? fp32 : 1.0f);
    }
    float rounds(int64_t steps, int kind) const { return round[kind] * ((steps + NW - 1) / NW); }
};
constexpr float kNot = 1e30f;
constexpr Cost costs[] = {{1, 1, 2.0f, 1.03f, {0.09f, 0.15f, 0.3f}, {0.57f, 1.6f, 1.9f}, {0.042f, 0.135f, 0.17f}},
                          {1, 2, 2.1f, 1.08f, {0.15f, 0.15f, 0.3f}, {0.62f, 1.5f, 1.85f}, {0.06f, 0.165f, 0.22f}},
                          {1, 4, 2.3f, 1.0f, {kNot, 0.25f, 0.2f}, {kNot, 1.9f, 2.6f}, {kNot, 0.2f, 0.37f}},
                          {1, 8, 2.6f, 1.0f, {kNot, 1.1f, 1.1f}, {kNot, 1.7f, 2.4f}, {kNot, 0.21f, 0.33f}},
                          {2, 2, 2.1f, 1.05f, {0.35f, kNot, kNot}, {0.88f, kNot, kNot}, {0.085f, kNot, kNot}},
                          {4, 4, 2.2f, 1.3f, {1.6f, kNot, kNot}, {1.2f, kNot, kNot}, {0.205f, kNot, kNot}}};
}  // namespace

Fp8Cut fp8_split_cut(int64_t m, int64_t n, int64_t steps, const hq_dtype *in, hq_dtype out) {
    const int kind = !in ? 0 : *in == HQ_F32 ? 2 : 1;
    const float cu = static_cast<float>(compute_units());
    Fp8Cut best{1, 1, 1e30f};
    for (const Cost &c : costs) {
        if ((m + 16 * c.mt - 1) / (16 * c.mt) > 65535) continue;   // (the grid's limit in y)
        // Fewer workgroups than CUs: each has a CU of its own.  Those that quantise keep a CU's vector units busy, so that a second one
        // on it waits (333 x 1024 -> 768, 252 of them, 4.5 us, 512 x 1024 -> 1024, 512, 6.1); those on codes wait for loads.  64 x 64 and
        // 16 x 128 fill a CU's LDS: no more than one for each CU (2048 x 3840 -> 960, 480 of 64 x 64, 24 us, 64 x 128 tiles 16; 1024 x
        // 1024 -> 1024, 512 of 16 x 128, 9.9, two launches 7.7).
        const float groups = static_cast<float>(c.groups(m, n)) / cu;
        float share = kind ? ceilf(groups) : std::max(groups, 1.0f);
        // (32 x 32 in eight waves: LDS for two on a CU, and a last round that is partly filled takes as long; 1429 x 2543 -> 393, 585 of
        // them, 12.5 us)
        if (c.mt == 2 && groups > 2.0f && 3 * std::min<int64_t>(NW, steps) * wave_bytes(2, 2) > kLdsPerCu)
            share = 2.0f * ceilf(groups / 2.0f);
        if (groups > 1.0f && 2 * NW * wave_bytes(c.mt, c.nt) > kLdsPerCu) continue;
        const float us = c.begin + std::max(c.rounds(steps, kind), share * c.workgroup(steps, kind, out));
        if (us < best.us) best = {c.mt, c.nt, us};
    }
    return best;
}

Fp8Cut fp8_split_pair_cut(const Fp8Product &a, const Fp8Product &b, hq_dtype out) {
    const float cu = static_cast<float>(compute_units());
    Fp8Cut best{1, 1, 1e30f};
    for (const Cost &c : costs) {
        if (c.mt > 2 || c.groups(a.m, a.n) + c.groups(b.m, b.n) > 0x3FFFFFFF) continue;
        const float one = c.workgroup(a.steps, 0, out, true), other = c.workgroup(b.steps, 0, HQ_F32, true);
        const float share = (static_cast<float>(c.groups(a.m, a.n)) * one + static_cast<float>(c.groups(b.m, b.n)) * other) / cu;
        const float us = c.begin + std::max(c.rounds(std::max(a.steps, b.steps), 0), std::max(share, std::max(one, other)));
        if (us < best.us) best = {c.mt, c.nt, us};
    }
    return best;
}

hq_status fp8_split_pair(const Fp8Product &a, const Fp8Product &b, const Fp8Sums &sums, Fp8Cut cut, hq_dtype out, hipStream_t st) {
    const SplitArgs x{a, nullptr, 0, 0}, y{b, nullptr, 0, 0};
    return out == HQ_F16 ? pair_with_cut<HQ_F16>(x, y, sums, cut, st) : out == HQ_BF16 ? pair_with_cut<HQ_BF16>(x, y, sums, cut, st)
                                                                                      : pair_with_cut<HQ_F32>(x, y, sums, cut, st);
}

hq_status fp8_split(const Fp8Product &p, Fp8Cut cut, const void *x, hq_dtype x_dtype, int64_t row_stride, int k, hq_dtype out,
                    hipStream_t st) {
    const SplitArgs a{p, x, row_stride, k};
    if (!x) return with_out<kCodes>(a, cut, out, st);
    switch (x_dtype) {
        case HQ_F16: return with_out<HQ_F16>(a, cut, out, st);
        case HQ_BF16: return with_out<HQ_BF16>(a, cut, out, st);
        default: return with_out<HQ_F32>(a, cut, out, st);
    }
}

}  // namespace hq
