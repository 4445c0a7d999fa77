// Product of E4M3 codes with block scales (hq_fp8.h):
//
//     y[i, j] = sum over blocks b of 128 of  sx[b, i] sw[j / 128, b] (sum over c in b of xq[i, c] wq[j, c])  + bias[j]
//
// The outer sum is fp32 fused multiply-adds.  The inner one is taken by matrix instructions started from zero, for results of 16 bits by one
// of 8-bit floats (16 x 16 x 128).  That instruction adds 8 neighbouring products after aligning them to the largest and keeps 13 bits
// below it, then goes on in fp32 (measured: a product 2^-13 as large as its neighbour counts, one 2^-14 as large is lost; between eights nothing
// is lost down to 2^-23).  Over normal values the sums are off by 2^-19 of the sum of magnitudes, far below what rounding to 16 bits takes, but not
// what fp32 sums give: fp32 results (weight gradients among them) use the bf16 instruction, which holds products of codes exactly and adds them
// in fp32, at half the rate.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cstdlib>

#include "hq_buffer.h"
#include "hq_common.h"
#include "hq_floats.h"
#include "hq_fp8.h"
#include "hq_fp6.h"

namespace {

constexpr int kStep = hq::kFp8Group;   // bytes of a row in one step, and values that share a scale

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct ProductArgs {
    const uint8_t *x, *w;        // codes [m, pitch], [n, pitch]
    const float *sx, *sw;        // [steps, m]; sw[block of channels * sw_block + step * sw_step]
    const void *bias;            // [n] of the output type, or null
    void *y;                     // [m, n]
    int64_t m;
    int n, pitch, steps;
    int sw_block, sw_step;
};

__device__ __forceinline__ f32x4 mfma_fp8(const v8i &a, const v8i &b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// A lane's 32 codes of a step as an operand of the 8-bit instruction, or of four bf16 ones (E4M3 numbers are bf16 numbers).
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <bool FP32> struct Operand {
    v8i v;
    __device__ __forceinline__ void set(const v4i &lo, const v4i &hi) { v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
};
template <> struct Operand<true> {
    bf16x8 v[4];
    __device__ __forceinline__ void set(const v4i &lo, const v4i &hi) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = static_cast<uint32_t>(i < 4 ? lo[i] : hi[i - 4]);
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
            const int at = (i & 1) * 4;
            v[i / 2][at] = a[0], v[i / 2][at + 1] = a[1], v[i / 2][at + 2] = b[0], v[i / 2][at + 3] = b[1];
        }
    }
};

// A tile of BM tokens x BN channels; WM x WN waves.  Codes of one step, [row][8 pieces of 16 bytes], go from memory straight into LDS;
// the pieces of a row are kept in an order that depends on the row, so that the 16 lanes of an LDS access read different banks (16 rows, two to a
// line of the 64 banks: 8 cycles a read of 16 bytes a lane without it, 4 with it).  Rows of weights are kept so that a lane's channels in NG tiles of results are
// neighbours.
// Two buffers.  The loads are written out: of the compiler's own it cannot tell which buffer they fill, and would let every read of LDS wait for
// all of them.  They have no register for a result; a wave waits for its own before the barrier that hands the buffer over.
__device__ __forceinline__ v4i words_of(const void *p, uint32_t bytes) {   // of a buffer's descriptor
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return v4i{static_cast<int>(at), static_cast<int>(at >> 32), static_cast<int>(bytes), 0x00027000};
}
// lane i's 16 (4) bytes to lds + 16 i (4 i); zeros from beyond the buffer
__device__ __forceinline__ void load16_to_lds(const v4i &buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void load4_to_lds(const v4i &buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "s"(lds) : "memory", "m0");
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
struct Product {
    using Out = typename Float<OUT>::type;
    static constexpr bool kFp32 = OUT == HQ_F32;
    static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    static constexpr int NG = NT < 4 ? NT : 4;   // a lane's neighbouring channels: 4 NG
    static constexpr int kCodes = (BM + BN) * kStep, LX = BM / 8 / NW, LW = BN / 8 / NW;
    // after the codes: the tokens' scales, then those of the blocks of channels, 64 copies of each
    static constexpr int SX = (BM + 63) / 64, SW = (BN + kStep - 1) / kStep, kTile = kCodes + (SX + SW) * 256;
    static constexpr int LS = (SX + SW + NW - 1) / NW, kLoads = LX + LW + LS;   // of a wave and step
    static_assert(LX >= 1 && LW >= 1 && (NW * 8) % 16 == 0, "whole loads; the order of pieces is the same in all loads of a wave");

    __device__ static __forceinline__ int key(int row) { return row >> 1 & 7; }
    // the channel that a row of LDS holds
    __host__ __device__ static constexpr int channel(int row) {
        return row / (16 * NG) * (16 * NG) + (row >> 2 & 3) * (4 * NG) + row / 16 % NG * 4 + (row & 3);
    }

    const ProductArgs &a;
    int lane, l16, quarter, wave, wm, wn, n0;
    int64_t m0;
    v4i xb, wb;
    uint32_t off_x, off_w, piece, at = 0;   // of the lane's next loads
    uint32_t ox, ow;                        // (beyond the buffer for a piece beyond the rows' end)
    uint32_t sx_bytes;
    uint32_t x_at[2], w_at[2], s_at;   // of the lane's two pieces of its first rows, and of its first scale, in a buffer
    f32x4 acc[NT][MT];

    __device__ __forceinline__ Product(const ProductArgs &args, uint32_t tile_m, uint32_t tile_n) : a(args) {
        const int tid = threadIdx.x;
        lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
        wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM;
        m0 = static_cast<int64_t>(tile_m) * BM, n0 = static_cast<int>(tile_n) * BN;
        const int rows_x = a.m - m0 < BM ? static_cast<int>(a.m - m0) : BM, rows_w = a.n - n0 < BN ? a.n - n0 : BN;
        xb = words_of(a.x + m0 * a.pitch, static_cast<uint32_t>(rows_x) * a.pitch);
        wb = words_of(a.w + static_cast<int64_t>(n0) * a.pitch, static_cast<uint32_t>(rows_w) * a.pitch);
        // a wave's load brings 8 rows: lane = (row, piece)
        const int row = wave * 8 + (lane >> 3);
        piece = ((lane & 7) ^ key(row)) * 16;
        off_x = static_cast<uint32_t>(row) * a.pitch + piece, off_w = static_cast<uint32_t>(channel(row)) * a.pitch + piece;
        sx_bytes = static_cast<uint32_t>(rows_x) * 4;
        const uint32_t lx = wm * TM + l16, lw = BM + wn * TN + l16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x_at[h] = lx * kStep + ((quarter * 2 + h) ^ key(lx)) * 16;
            w_at[h] = lw * kStep + ((quarter * 2 + h) ^ key(lw)) * 16;
        }
        s_at = kCodes + lx * 4;
        // (the compiler would otherwise keep an address for every read: it cannot tell that the offsets add without a carry)
        asm("" : "+v"(x_at[0]), "+v"(x_at[1]), "+v"(w_at[0]), "+v"(w_at[1]), "+v"(s_at));
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Requests the codes and scales of the next step for the buffer at `lds`, in kLoads parts.
    __device__ __forceinline__ void begin_request() {
        const bool inside = at + piece < static_cast<uint32_t>(a.pitch);   // (the last step may end inside)
        ox = inside ? off_x : 0x80000000u, ow = inside ? off_w : 0x80000000u;
        off_x += kStep, off_w += kStep, at += kStep;
    }
    __device__ __forceinline__ void request_part(int part, uint32_t lds, int step) const {
        if (part < LX) {
            load16_to_lds(xb, ox + static_cast<uint32_t>(part * NW * 8) * a.pitch, lds + (part * NW + wave) * 1024);
        } else if (part < LX + LW) {
            const int l = part - LX;
            load16_to_lds(wb, ow + static_cast<uint32_t>(channel(l * NW * 8)) * a.pitch, lds + (BM / 8 + l * NW + wave) * 1024);
        } else {
            // (waves without a piece of their own repeat the last one: all count the same loads)
            const int l = part - LX - LW, i = l * NW + wave < SX + SW ? l * NW + wave : SX + SW - 1;
            const bool tokens = i < SX;
            // (channels of a tile beyond the last block are not stored)
            const int block = n0 / kStep + i - SX, last = (a.n - 1) / kStep;
            const float *from = tokens ? a.sx + static_cast<int64_t>(step) * a.m + m0
                                       : a.sw + static_cast<int64_t>(block < last ? block : last) * a.sw_block + static_cast<int64_t>(step) * a.sw_step;
            load4_to_lds(words_of(from, tokens ? sx_bytes : 4), tokens ? (i * 64 + lane) * 4 : 0, lds + kCodes + i * 256);
        }
    }
    __device__ __forceinline__ void request(uint32_t lds, int step) {
        begin_request();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) request_part(i, lds, step);
    }
    // The wave's loads for this step have landed (those for the AHEAD steps after it may be under way), and so have the others'; all
    // have read the buffer that is filled next.
    template <int AHEAD> __device__ __forceinline__ static void hand_over() {
        static_assert(AHEAD * kLoads < 64, "the counter of loads has 6 bits");
        wait_vmem<AHEAD * kLoads>();
        lds_barrier();
    }

    __device__ __forceinline__ static void fetch(Operand<kFp32> &o, const uint8_t *lo, const uint8_t *hi) {
        o.set(*reinterpret_cast<const v4i *>(lo), *reinterpret_cast<const v4i *>(hi));
    }
    __device__ __forceinline__ void fetch_w(Operand<kFp32> &o, const uint8_t *lds, int i) const {
        const int skip = i * 16 * kStep;
        fetch(o, lds + w_at[0] + skip, lds + w_at[1] + skip);
    }

    // One step from LDS.  The products of a row of tiles are folded into the sums beside the products of the next row; the loads of step `ahead`
    // (if REQUEST) are dealt over the rows, since a wave that issues them all at once waits for the path to memory.
    template <bool REQUEST> __device__ __forceinline__ void step(const uint8_t *lds, uint32_t fill = 0, int ahead = 0) {
        if constexpr (REQUEST) begin_request();
        Operand<kFp32> x[MT], w[2];
        float s[MT];
        const float s_w = *reinterpret_cast<const float *>(lds + kCodes + (SX + wn * TN / kStep) * 256);
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            fetch(x[j], lds + x_at[0] + j * 16 * kStep, lds + x_at[1] + j * 16 * kStep);
            s[j] = *reinterpret_cast<const float *>(lds + s_at + j * 64) * s_w;
        }
        fetch_w(w[0], lds, 0);
        f32x4 p[MT];
#pragma unroll
        for (int i = 0; i <= NT; ++i) {
            if (i + 1 < NT) fetch_w(w[(i + 1) & 1], lds, i + 1);
            if constexpr (REQUEST) {
#pragma unroll
                for (int part = i * kLoads / NT; part < (i + 1) * kLoads / NT && i < NT; ++part) request_part(part, fill, ahead);
            }
            if constexpr (!kFp32) {
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    if (i > 0) fold(i - 1, j, p[j], s[j]);
                    if (i < NT) p[j] = mfma_fp8(w[i & 1].v, x[j].v);
                }
                // four multiply-adds of the row before, a product, in this order
                if (i + 1 < NT) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    if (i > 0) __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                    if (i < NT) __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            } else {
                f32x4 q[MT];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < MT; ++j) {
                        if (i < NT)
                            q[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i & 1].v[k], x[j].v[k], k ? q[j] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                        if (i > 0 && k == 0) fold(i - 1, j, p[j], s[j]);
                    }
#pragma unroll
                for (int j = 0; j < MT; ++j) p[j] = q[j];
            }
        }
    }
    __device__ __forceinline__ void fold(int i, int j, const f32x4 &p, float s) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], s, acc[i][j][e]);
    }

    // Results: a lane has 4 NG neighbouring channels of a token.
    __device__ __forceinline__ void store() const {
        constexpr int CH = 4 * NG;
#pragma unroll
        for (int g = 0; g < NT / NG; ++g) {
            const int c = n0 + wn * TN + g * 16 * NG + quarter * CH;
            const bool whole = c + CH <= a.n;
            float bias[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) bias[e] = 0.0f;
            if (a.bias) {
                const Out *b = static_cast<const Out *>(a.bias);
#pragma unroll
                for (int e = 0; e < CH; ++e) bias[e] = static_cast<float>(b[c + e < a.n ? c + e : a.n - 1]);
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const int64_t t = m0 + wm * TM + j * 16 + l16;
                if (t >= a.m) continue;
                Out *y = static_cast<Out *>(a.y) + t * a.n + c;
                typename Vec<Out, CH>::type v;
#pragma unroll
                for (int e = 0; e < CH; ++e) v[e] = round_to<Out>(acc[g * NG + e / 4][j][e % 4] + bias[e]);
                if (whole) {
                    store_vec<Out, CH>(y, v);
                } else {
#pragma unroll
                    for (int e = 0; e < CH; ++e)
                        if (c + e < a.n) y[e] = v[e];
                }
            }
        }
    }
};

// Neighbouring workgroups share tiles' codes in the L2 of their XCD: workgroup b runs on XCD b % 8, each XCD takes a contiguous run of tiles,
// and those go through bands of 4 tiles of tokens.
struct Tiles {
    uint32_t m, n;   // counts
};
__device__ __forceinline__ Tiles tile_of(uint32_t b, Tiles count) {
    const uint32_t all = count.m * count.n, xcd = b & 7, q = all >> 3, r = all & 7;
    const uint32_t t = xcd * q + (xcd < r ? xcd : r) + (b >> 3);
    const uint32_t band = t / (4 * count.n), in = t - band * 4 * count.n, left = count.m - band * 4, high = left < 4 ? left : 4;
    return {band * 4 + in % high, in / high};
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN * 64) void product_kernel(ProductArgs a, Tiles count) {
    using P = Product<OUT, BM, BN, WM, WN, STAGES>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const uint32_t lds_at = lds_address(lds);
    const Tiles tile = tile_of(blockIdx.x, count);
    P p(a, tile.m, tile.n);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < a.steps) p.request(lds_at + i * P::kTile, i);
    uint32_t now = 0, next = (STAGES - 1) * P::kTile;   // the buffers that are read and filled
    const auto turn = [&] {
        next = now;
        now = now + P::kTile < STAGES * P::kTile ? now + P::kTile : 0;
    };
    int i = 0;
    for (; i + STAGES - 1 < a.steps; ++i) {
        P::template hand_over<STAGES - 2>();
        p.template step<true>(lds + now, lds_at + next, i + STAGES - 1);
        turn();
    }
    for (; i < a.steps; ++i) {
        P::template hand_over<0>();
        p.template step<false>(lds + now);
        turn();
    }
    p.store();
}

__global__ __launch_bounds__(256) void zero_kernel(float *p, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) p[i] = 0.0f;
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
hq_status launch_tiles(const ProductArgs &a, hipStream_t st) {
    const Tiles count{static_cast<uint32_t>((a.m + BM - 1) / BM), static_cast<uint32_t>((a.n + BN - 1) / BN)};
    constexpr auto kernel = product_kernel<OUT, BM, BN, WM, WN, STAGES>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    const hq::LaunchCheck check;
    kernel<<<count.m * count.n, WM * WN * 64, STAGES * Product<OUT, BM, BN, WM, WN, STAGES>::kTile, st>>>(a, count);
    return check.status();
}

template <int OUT>
hq_status launch(const ProductArgs &a, hipStream_t st) {
    static const int force = getenv("HQ_TILE") ? atoi(getenv("HQ_TILE")) : -1;
    switch (force) {
        case 0: if constexpr (OUT != HQ_F32) return launch_tiles<OUT, 256, 256, 4, 2, 2>(a, st); else return launch_tiles<OUT, 256, 128, 4, 2, 2>(a, st);
        case 1: return launch_tiles<OUT, 128, 128, 2, 2, 2>(a, st);
        case 2: return launch_tiles<OUT, 128, 128, 2, 2, 4>(a, st);
        case 3: return launch_tiles<OUT, 64, 128, 2, 2, 3>(a, st);
        case 4: return launch_tiles<OUT, 64, 128, 2, 2, 6>(a, st);
        case 5: return launch_tiles<OUT, 64, 64, 2, 2, 4>(a, st);
        case 6: return launch_tiles<OUT, 256, 128, 4, 2, 2>(a, st);
        case 7: return launch_tiles<OUT, 256, 128, 4, 2, 3>(a, st);
        case 8: return launch_tiles<OUT, 128, 128, 2, 4, 4>(a, st);
        case 9: return launch_tiles<OUT, 128, 128, 2, 4, 2>(a, st);
        case 10: return launch_tiles<OUT, 128, 256, 2, 2, 2>(a, st);
        case 11: return launch_tiles<OUT, 64, 64, 2, 2, 8>(a, st);
        case 12: return launch_tiles<OUT, 128, 256, 2, 4, 3>(a, st);
    }
    const int64_t large = ((a.m + 255) / 256) * ((a.n + 255) / 256);
    if constexpr (OUT != HQ_F32) {
        if (large >= 200) return launch_tiles<OUT, 256, 256, 4, 2, 2>(a, st);
    }
    return launch_tiles<OUT, 128, 128, 2, 2, 2>(a, st);
}

hq_status product(const uint8_t *xq, const float *x_scale, const uint8_t *wq, const float *w_scale, bool scale_turned, const void *bias,
                  int64_t m, int n, int k, void *y, hq_dtype dt, hipStream_t st) {
    const int steps = static_cast<int>(hq::fp8_groups(k));
    const int blocks = static_cast<int>(hq::fp8_groups(n));
    const ProductArgs a{xq, wq, x_scale, w_scale, bias, y, m, n, hq::fp8_pitch(k), steps, scale_turned ? 1 : steps, scale_turned ? blocks : 1};
    switch (dt) {
        case HQ_F16: return launch<HQ_F16>(a, st);
        case HQ_BF16: return launch<HQ_BF16>(a, st);
        case HQ_F32: return launch<HQ_F32>(a, st);
        default: return HQ_ERR_DTYPE;
    }
}

// Rows of codes whose tiles are addressed with 31-bit offsets, and tile counts that fit a grid.
bool product_fits(int64_t m, int64_t n, int64_t k) {
    return k <= (int64_t{1} << 31) / 256 - 16 && ((m + 15) / 16) * ((n + 15) / 16) <= 0x7FFFFFFF;
}

int64_t up256(int64_t v) { return (v + 255) & ~int64_t{255}; }

// the workspace of a backward pass, in bytes from its start
struct BackwardSpace {
    int64_t dyq, dyq_t, xq_t, dy_scale, dy_scale_t, x_scale, sums, total;
    BackwardSpace(int64_t m, int64_t n, int64_t k) {
        int64_t at = 0;
        const auto take = [&](int64_t bytes) {
            const int64_t here = at;
            at += up256(bytes);
            return here;
        };
        dyq = take(m * hq::fp8_pitch64(n));
        dyq_t = take(n * hq::fp8_pitch64(m));
        xq_t = take(k * hq::fp8_pitch64(m));
        dy_scale = take(4 * hq::fp8_groups(n) * m);
        dy_scale_t = take(4 * hq::fp8_groups(m) * n);
        x_scale = take(4 * hq::fp8_groups(m) * hq::fp8_groups(k));
        sums = take(4 * hq::fp8_groups(m) * n);
        total = at;
    }
};

}  // namespace

extern "C" hq_status hq_fp8_linear(const uint8_t *xq, const float *x_scale, const uint8_t *wq, const float *w_scale, int w_scale_turned,
                                   const void *bias, int64_t m, int n, int k, void *y, hq_dtype y_dtype, void *stream) {
    if (!wq || !w_scale || (m > 0 && (!xq || !x_scale || !y))) return HQ_ERR_NULL;
    if (!hq::is_float(y_dtype)) return HQ_ERR_DTYPE;
    if (m < 0 || n <= 0 || k <= 0) return HQ_ERR_SHAPE;
    const int size = hq::size_of(y_dtype);
    if (!hq::aligned16(xq) || !hq::aligned16(wq) || !hq::aligned_to(x_scale, 4) || !hq::aligned_to(w_scale, 4) ||
        !hq::aligned_to(y, size) || !hq::aligned_to(bias, size))
        return HQ_ERR_ALIGN;
    if (!product_fits(m, n, k)) return HQ_ERR_UNSUPPORTED;
    if (m == 0) return HQ_OK;
    return product(xq, x_scale, wq, w_scale, w_scale_turned != 0, bias, m, n, k, y, y_dtype, static_cast<hipStream_t>(stream));
}

extern "C" int64_t hq_act_quant_fp8_linear_workspace(int64_t m, int k) {
    if (m <= 0 || k <= 0) return 0;
    return up256(m * hq::fp8_pitch64(k)) + up256(4 * hq::fp8_groups(k) * m);
}

extern "C" hq_status hq_act_quant_fp8_linear(const void *x, hq_dtype x_dtype, int64_t row_stride, const uint8_t *wq, const float *w_scale,
                                             const void *bias, int64_t m, int n, int k, void *workspace, void *y, hq_dtype y_dtype,
                                             void *stream) {
    if (!wq || !w_scale || (m > 0 && (!x || !y || !workspace))) return HQ_ERR_NULL;
    if (!hq::is_float(x_dtype) || !hq::is_float(y_dtype)) return HQ_ERR_DTYPE;
    if (m < 0 || n <= 0 || k <= 0 || row_stride < 0) return HQ_ERR_SHAPE;
    const int size = hq::size_of(y_dtype);
    if (!hq::aligned_to(x, hq::size_of(x_dtype)) || !hq::aligned16(wq) || !hq::aligned_to(w_scale, 4) || !hq::aligned16(workspace) ||
        !hq::aligned_to(y, size) || !hq::aligned_to(bias, size))
        return HQ_ERR_ALIGN;
    if (!product_fits(m, n, k) || !hq::fp8_fits(m, k)) return HQ_ERR_UNSUPPORTED;
    if (m == 0) return HQ_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint8_t *xq = static_cast<uint8_t *>(workspace);
    float *sx = reinterpret_cast<float *>(xq + up256(m * hq::fp8_pitch64(k)));
    if (const hq_status s = hq::fp8_rows(x, x_dtype, m, k, row_stride, xq, sx, st)) return s;
    return product(xq, sx, wq, w_scale, false, bias, m, n, k, y, y_dtype, st);
}

extern "C" int64_t hq_fp8_linear_backward_workspace(int64_t m, int n, int k) {
    if (m <= 0 || n <= 0 || k <= 0) return 0;
    return BackwardSpace(m, n, k).total;
}

extern "C" hq_status hq_fp8_linear_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, hq_dtype dtype,
                                            const uint8_t *wq_t, const float *w_scale, int64_t m, int n, int k, void *workspace, void *dx,
                                            float *dw, float *db, void *stream) {
    if (!wq_t || !w_scale || !dw || (m > 0 && (!dy || !x || !dx || !workspace))) return HQ_ERR_NULL;
    if (!hq::is_float(dtype)) return HQ_ERR_DTYPE;
    if (m < 0 || n <= 0 || k <= 0 || dy_stride < 0 || x_stride < 0) return HQ_ERR_SHAPE;
    const int size = hq::size_of(dtype);
    if (!hq::aligned_to(dy, size) || !hq::aligned_to(x, size) || !hq::aligned_to(dx, size) || !hq::aligned16(wq_t) ||
        !hq::aligned_to(w_scale, 4) || !hq::aligned16(workspace) || !hq::aligned_to(dw, 4) || !hq::aligned_to(db, 4))
        return HQ_ERR_ALIGN;
    if (!product_fits(m, k, n) || !product_fits(n, k, m) || !hq::fp8_fits(m, n) || !hq::fp8_fits(m, k)) return HQ_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (m == 0) {
        const hq::LaunchCheck check;
        zero_kernel<<<std::min<uint32_t>(1024, (static_cast<int64_t>(n) * k + 255) / 256), 256, 0, st>>>(dw, static_cast<int64_t>(n) * k);
        if (db) zero_kernel<<<std::min<uint32_t>(1024, (n + 255) / 256), 256, 0, st>>>(db, n);
        return check.status();
    }
    uint8_t *base = static_cast<uint8_t *>(workspace);
    const BackwardSpace at(m, n, k);
    const auto f32 = [&](int64_t offset) { return reinterpret_cast<float *>(base + offset); };
    if (const hq_status s = hq::fp8_both(dy, dtype, m, n, dy_stride, base + at.dyq, f32(at.dy_scale), base + at.dyq_t, f32(at.dy_scale_t),
                                         f32(at.sums), db, st))
        return s;
    if (const hq_status s = hq::fp8_blocks(x, dtype, m, k, x_stride, nullptr, base + at.xq_t, f32(at.x_scale), st)) return s;
    // dx [m, k] = dy [m, n] W [n, k]: the weights' codes with rows of n, their scales as those of W
    if (const hq_status s = product(base + at.dyq, f32(at.dy_scale), wq_t, w_scale, true, nullptr, m, k, n, dx, dtype, st)) return s;
    // dW [n, k] = dy^T [n, m] x [m, k]
    return product(base + at.dyq_t, f32(at.dy_scale_t), base + at.xq_t, f32(at.x_scale), true, nullptr, n, k, static_cast<int>(m), dw,
                   HQ_F32, st);
}
