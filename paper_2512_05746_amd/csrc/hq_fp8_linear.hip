// Product of E4M3 codes with block scales (hq_fp8.h):
//
//     y[i, j] = sum over blocks b of 128 of  sx[b, i] sw[j / 128, b] (sum over c in b of xq[i, c] wq[j, c])  + bias[j]
//
// The outer sum is fp32 fused multiply-adds.  The inner one is taken by matrix instructions started from zero, for results of 16 bits by
// one of 8-bit floats (16 x 16 x 128).  That instruction cuts 8 neighbouring products towards zero to multiples of 2^(e - 13), e the
// largest sum of two exponents among those that are not zero (subnormal codes count -6), and adds them in fp32 (measured on single
// products, and sums of 128 .. 4096 of normal values agree with this in every fp16 result).  At most 7 products of an eight lose 2^-13 of
// the largest, 2^-10 of the sum of magnitudes, or 8 times that where the largest is a subnormal code's.  Over normal values the results
// are off by 1.5e-5 of their norm (fp16 rounding: 2.1e-4) and 6 % of fp16 results are the neighbour of the nearest one: taken for twice
// the rate.  Not for fp32 results (weight gradients among them): they use the bf16 instruction, which holds products of codes exactly and
// adds them in fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "hq_buffer.h"
#include "hq_common.h"
#include "hq_floats.h"
#include "hq_fp8.h"
#include "hq_fp8_product.h"

namespace {

// A tile of BM tokens x BN channels; WM x WN waves.  Codes of one step, [row][8 pieces of 16 bytes], go from memory straight into LDS;
// the pieces of a row are kept in an order that depends on the row, so that lanes that are served together read different banks.  Rows of
// weights are kept so that a lane's channels in NG tiles of results are neighbours.
//
// A wave takes the products of a step in a fixed order, each with the fold of the one four before it (the multiply-adds issue while
// the matrix pipe is busy): rows of its tiles, the last two rows together, column by column.  Each operand is read from LDS two rows
// ahead, and the tokens' operands of the next step as soon as the last product with their predecessor has been issued, so that no step
// begins with a wait.  The one barrier of a step stands before the last two rows: there all waves have read the buffer of this step,
// which is then filled again, and the buffer of the next one has landed.  The loads of a step are dealt over the products, since a wave
// that issues them all at once waits for the path to memory.
//
// (The loads have to be those of hq_fp8_product.h, which the compiler does not wait for.)
//
// What bounds it: 8192 x 4096 -> 8192 with 256 x 256 tiles 239 us (2.3 PFLOP/s; a library product of the same codes with one scale for
// the tensor 229 .. 231): the matrix pipe is busy in 62 % of the cycles and the clock is at 1.73 of 2.4 GHz, so it is power; at few
// workgroups LDS (192 KB of reads and 64 KB of loads a step, 128 bytes a cycle, against 2048 cycles of the matrix pipe).  fp32 results:
// 4096 x 8192 -> 4096 239 us (1.15 PFLOP/s; bf16 products of a library 1.42).  Small K (4096 x 576 -> 1728 12.2 us, 8.2 with K = 128):
// launch, first loads and results (14 MB) of one round of workgroups.
template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
struct Product {
    using Out = typename Float<OUT>::type;
    static constexpr bool kFp32 = OUT == HQ_F32;
    static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    // A lane's neighbouring channels, 4 NG, are the 16 bytes of a store: the 4 lanes of a token then write 64 bytes in a row.
    static constexpr int NG = kFp32 ? 1 : 2;
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

    static constexpr int T = MT * NT, kBody = (NT - 2) * MT, RING = 4;   // products of a step, those before the last two rows
    static_assert(T >= RING && MT % 2 == 0 && (NT == 2 || NT % 4 == 0), "the order of the products");
    __host__ __device__ static constexpr int row_of(int t) { return t < kBody ? t / MT : NT - 2 + ((t - kBody) & 1); }
    __host__ __device__ static constexpr int column_of(int t) { return t < kBody ? t % MT : (t - kBody) / 2; }

    const ProductArgs &a;
    int lane, l16, quarter, wave, wm, wn, n0;
    int64_t m0;
    v4i xb, wb;
    uint32_t off_x, off_w, piece;            // of the lane's next loads
    uint32_t ox, ow;                         // (beyond the buffer for a piece beyond the rows' end)
    uint32_t fill, sx_bytes;
    int requested = 0;                       // steps
    uint32_t x_at[2], w_at[2], s_at;         // of the lane's two pieces of its first rows, and of its first scale, in a buffer
    v8i x[MT], w[4];
    f32x4 acc[NT][MT], p[RING];
    // scales of this step, of the columns whose products of the step before are not folded yet, of the next step
    float s[MT], s_old[2], s_new[MT], s_w;

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
#pragma unroll
        for (int i = 0; i < RING; ++i) p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        s_old[0] = s_old[1] = 0.0f;
    }

    // Requests the codes and scales of the next step for the buffer at `lds`, in kLoads parts.  Beyond the last step: zeros from beyond the
    // buffers, so that all steps count the same loads.
    __device__ __forceinline__ void begin_request(uint32_t lds) {
        fill = lds;
        const bool inside = requested * kStep + static_cast<int>(piece) < a.pitch;   // (the last step may end inside)
        ox = inside ? off_x : 0x80000000u, ow = inside ? off_w : 0x80000000u;
        off_x += kStep, off_w += kStep, ++requested;
    }
    __device__ __forceinline__ void request_part(int part) const {
        if (part < LX) {
            load16_to_lds(xb, ox + static_cast<uint32_t>(part * NW * 8) * a.pitch, fill + (part * NW + wave) * 1024);
        } else if (part < LX + LW) {
            const int l = part - LX;
            load16_to_lds(wb, ow + static_cast<uint32_t>(channel(l * NW * 8)) * a.pitch, fill + (BM / 8 + l * NW + wave) * 1024);
        } else {
            // (waves without a piece of their own repeat the last one)
            const int l = part - LX - LW, i = l * NW + wave < SX + SW ? l * NW + wave : SX + SW - 1, step = requested - 1;
            const bool tokens = i < SX;
            // (channels of a tile beyond the last block are not stored)
            const int block = n0 / kStep + i - SX, last = (a.n - 1) / kStep;
            const float *from = tokens ? a.sx + static_cast<int64_t>(step) * a.m + m0
                                       : a.sw + static_cast<int64_t>(block < last ? block : last) * a.sw_block +
                                             static_cast<int64_t>(step) * a.sw_step;
            load4_to_lds(words_of(from, step >= a.steps ? 0 : tokens ? sx_bytes : 4), tokens ? (i * 64 + lane) * 4 : 0,
                         fill + kCodes + i * 256);
        }
    }
    __device__ __forceinline__ void request(uint32_t lds) {
        begin_request(lds);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) request_part(i);
    }
    // All but the wave's last LATER loads have landed, and so have the others'; all have read what is filled next.
    template <int LATER> __device__ __forceinline__ static void hand_over() {
        wait_vmem<LATER>();
        lds_barrier();
    }

    __device__ __forceinline__ static v8i fetch(const uint8_t *lo, const uint8_t *hi) {
        return __builtin_shufflevector(*reinterpret_cast<const v4i *>(lo), *reinterpret_cast<const v4i *>(hi), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ void fetch_x(const uint8_t *lds, int j) {
        x[j] = fetch(lds + x_at[0] + j * 16 * kStep, lds + x_at[1] + j * 16 * kStep);
    }
    __device__ __forceinline__ void fetch_w(const uint8_t *lds, int i) {
        w[i & 3] = fetch(lds + w_at[0] + i * 16 * kStep, lds + w_at[1] + i * 16 * kStep);
    }
    __device__ __forceinline__ void fetch_scales(const uint8_t *lds) {
        s_w = *reinterpret_cast<const float *>(lds + kCodes + (SX + wn * TN / kStep) * 256);
#pragma unroll
        for (int j = 0; j < MT; ++j) s_new[j] = *reinterpret_cast<const float *>(lds + s_at + j * 64);
    }
    __device__ __forceinline__ void take_scales() {
        s_old[0] = s[MT - 2], s_old[1] = s[MT - 1];
#pragma unroll
        for (int j = 0; j < MT; ++j) s[j] = s_new[j] * s_w;
    }
    // what the first step begins with
    __device__ __forceinline__ void begin(const uint8_t *lds) {
#pragma unroll
        for (int j = 0; j < MT; ++j) s[j] = 0.0f, fetch_x(lds, j);
        fetch_w(lds, 0);
        fetch_w(lds, 1);
        fetch_scales(lds);
        take_scales();
    }

    // adds the product that went into p[t % RING]; t < 0: of the step before
    __device__ __forceinline__ void fold(int t) {
        const int u = t < 0 ? t + T : t, i = row_of(u), j = column_of(u);
        const float scale = t < 0 ? s_old[j - (MT - 2)] : s[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[u % RING][e], scale, acc[i][j][e]);
    }
    __device__ __forceinline__ void finish() {   // (s_old holds the last step's)
#pragma unroll
        for (int t = -RING; t < 0; ++t) fold(t);
    }

    // reads that go with product t (of NT >= 4 rows)
    __device__ __forceinline__ void before(int t, const uint8_t *now, const uint8_t *next) {
        if (t < kBody && t % MT == 0) fetch_w(now, t / MT + 2);
        if constexpr (NT > 2) {
            if (t == kBody) fetch_w(next, 0);
            if (t == kBody + 2) fetch_w(next, 1);
        }
        if (t == T - 2) fetch_scales(next);
    }
    __device__ __forceinline__ void after(int t, const uint8_t *next) {
        if (t >= kBody && (t - kBody) % 2 == 1) fetch_x(next, column_of(t));
        if (NT == 2 && t >= T - 2) fetch_w(next, t - (T - 2));
    }
    // loads that go with product t: a request begins after the barrier and goes on in the next step
    static constexpr int OVER = T < 16 ? T : 16;
    static constexpr int kFirst = (2 * MT < OVER ? 2 * MT : OVER) * kLoads / OVER;   // parts of a request before the next step
    __device__ __forceinline__ void deal(int t) const {
        const int slot = t >= kBody ? t - kBody : t + 2 * MT;
        if (slot < OVER) {
#pragma unroll
            for (int part = slot * kLoads / OVER; part < (slot + 1) * kLoads / OVER; ++part) request_part(part);
        }
    }

    // One step from the buffer `now`, which is filled for a later step from its barrier on; `next` holds the step after it.
    template <int LATER> __device__ __forceinline__ void step(const uint8_t *now, const uint8_t *next, uint32_t now_at) {
        Halves xh[kFp32 ? MT : 1], wh[2];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if (t == kBody) {
                hand_over<LATER>();
                begin_request(now_at);
            }
            before(t, now, next);
            deal(t);
            const int i = row_of(t), j = column_of(t);
            if constexpr (!kFp32) {
                fold(t - RING);
                p[t % RING] = mfma_fp8(w[i & 3], x[j]);
                __builtin_amdgcn_sched_barrier(0);
                after(t, next);
            } else {
                // (converted once: the tokens' operands at the start of the step, those of the weights with their rows)
                if (t == 0) {
#pragma unroll
                    for (int c = 0; c < MT; ++c) xh[c] = halves_of(x[c]);
                }
                if (t < kBody ? t % MT == 0 : t == kBody) wh[0] = halves_of(w[i & 3]);
                if (t == kBody) wh[1] = halves_of(w[(NT - 1) & 3]);
                if (t % 2 == 1) {   // two products side by side: the four instructions of one wait for each other
                    const bool body = t < kBody;
                    fold(t - 1 - RING);
                    fold(t - RING);
                    f32x4 a0{0.f, 0.f, 0.f, 0.f}, a1{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        a0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wh[0].v[k], xh[column_of(t - 1)].v[k], a0, 0, 0, 0);
                        a1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wh[body ? 0 : 1].v[k], xh[j].v[k], a1, 0, 0, 0);
                    }
                    p[(t - 1) % RING] = a0, p[t % RING] = a1;
                    __builtin_amdgcn_sched_barrier(0);
                    after(t - 1, next);
                    after(t, next);
                }
            }
        }
        take_scales();
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

// Neighbouring workgroups share tiles' codes in the L2 of their XCD: workgroup b runs on XCD b % 8, each XCD takes a contiguous run of
// tiles, and those go through bands of 4 tiles of tokens.
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
__device__ __forceinline__ void product_tile(const ProductArgs &a, Tiles count, uint32_t block, uint8_t *lds) {
    using P = Product<OUT, BM, BN, WM, WN, STAGES>;
    const uint32_t lds_at = lds_address(lds);
    const Tiles tile = tile_of(block, count);
    P p(a, tile.m, tile.n);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) p.request(lds_at + i * P::kTile);
    p.begin_request(lds_at + (STAGES - 1) * P::kTile);
#pragma unroll
    for (int i = 0; i < P::kFirst; ++i) p.request_part(i);
    P::template hand_over<(STAGES - 2) * P::kLoads + P::kFirst>();
    p.begin(lds);
    uint32_t now = 0;
    for (int i = 0; i < a.steps; ++i) {
        const uint32_t next = now + P::kTile < STAGES * P::kTile ? now + P::kTile : 0;
        p.template step<(STAGES - 2) * P::kLoads>(lds + now, lds + next, lds_at + now);
        now = next;
    }
    p.finish();
    wait_vmem<0>();   // (nothing may land in LDS that the workgroup no longer owns)
    p.store();
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN * 64) void product_kernel(ProductArgs a, Tiles count) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    product_tile<OUT, BM, BN, WM, WN, STAGES>(a, count, blockIdx.x, lds);
}

// Two products, `b` with fp32 results, and sums: workgroups of b first, then of a, then of the sums.
template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN * 64) void product_pair_kernel(ProductArgs a, Tiles a_count, ProductArgs b, Tiles b_count,
                                                                   hq::Fp8Sums sums) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const uint32_t na = a_count.m * a_count.n, nb = b_count.m * b_count.n;
    if (blockIdx.x < nb) product_tile<HQ_F32, BM, BN, WM, WN, STAGES>(b, b_count, blockIdx.x, lds);
    else if (blockIdx.x < nb + na) product_tile<OUT, BM, BN, WM, WN, STAGES>(a, a_count, blockIdx.x - nb, lds);
    else sum_rows(sums, blockIdx.x - nb - na, threadIdx.x, reinterpret_cast<float *>(lds));
}
__global__ __launch_bounds__(256) void sum_rows_kernel(hq::Fp8Sums sums) {
    __shared__ float lds[256];
    sum_rows(sums, blockIdx.x, threadIdx.x, lds);
}

__global__ __launch_bounds__(256) void zero_kernel(float *p, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) p[i] = 0.0f;
}

template <int BM, int BN>
Tiles tiles_of(const ProductArgs &a) {
    return {static_cast<uint32_t>((a.m + BM - 1) / BM), static_cast<uint32_t>((a.n + BN - 1) / BN)};
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
hq_status launch_tiles(const ProductArgs &a, hipStream_t st) {
    const Tiles count = tiles_of<BM, BN>(a);
    constexpr auto kernel = product_kernel<OUT, BM, BN, WM, WN, STAGES>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    const hq::LaunchCheck check;
    kernel<<<count.m * count.n, WM * WN * 64, STAGES * Product<OUT, BM, BN, WM, WN, STAGES>::kTile, st>>>(a, count);
    return check.status();
}

template <int OUT, int BM, int BN, int WM, int WN, int STAGES>
hq_status launch_pair(const ProductArgs &a, const ProductArgs &b, const hq::Fp8Sums &sums, hipStream_t st) {
    const Tiles ca = tiles_of<BM, BN>(a), cb = tiles_of<BM, BN>(b);
    constexpr auto kernel = product_pair_kernel<OUT, BM, BN, WM, WN, STAGES>;
    static std::atomic<uint64_t> allowed;
    if (const hq_status s = allow_lds(reinterpret_cast<const void *>(kernel), allowed)) return s;
    constexpr int bytes = STAGES * std::max(Product<OUT, BM, BN, WM, WN, STAGES>::kTile, Product<HQ_F32, BM, BN, WM, WN, STAGES>::kTile);
    const hq::LaunchCheck check;
    kernel<<<ca.m * ca.n + cb.m * cb.n + sum_blocks(sums), WM * WN * 64, bytes, st>>>(a, ca, b, cb, sums);
    return check.status();
}

// The tiles of the product, for 16-bit results first, then for 32-bit ones.  A step of a lone workgroup takes `round` us, a CU's share of a
// step `each` us a tile when it has several; measured with 8192 x 4096 -> 8192 and 4096 x 8192 -> 4096 (shares), 2048 x 3840 -> 960, 1024
// x 1024 -> 1024 and 256 x 4096 -> 4096 (rounds); begin: launch, first loads and results (300 x 100 -> 4100, 1025 x 500 -> 1030), again:
// those of a CU's further tiles (2048 x 512 -> 2048, 4096 x 256 -> 1024).  Tiles of 128 x 128, two workgroups a CU, are not among them:
// 335 us for 8192 x 4096 -> 8192 where 256 x 128 takes 302 and 256 x 256 257; with fp32 results 246 us for 4096 x 8192 -> 4096 where 256
// x 128 takes 239 (the card's power is the limit there, and larger tiles move less through LDS).
enum Tile { kTile256, kTile128, kTile64x128, kTile64 };
struct TileCost {
    Tile tile;
    int bm, bn;
    float begin, again, round[2], each[2];
};
constexpr float kNot = 1e30f;
constexpr TileCost kTiles[] = {{kTile256, 256, 256, 7.0f, 0.0f, {1.4f, kNot}, {1.6f, kNot}},
                               {kTile128, 256, 128, 5.1f, 0.0f, {0.9f, 1.6f}, {1.18f, 1.87f}},
                               {kTile64x128, 64, 128, 3.3f, 0.5f, {0.44f, 0.8f}, {0.38f, 0.6f}},
                               {kTile64, 64, 64, 2.6f, 0.5f, {0.33f, 0.49f}, {0.24f, 0.38f}}};
struct TileChoice {
    Tile tile;
    float us;
};
// tiles a CU, in shares of a CU
float tiles_per_cu(const TileCost &c, int64_t m, int64_t n, float cu) {
    return static_cast<float>(((m + c.bm - 1) / c.bm) * ((n + c.bn - 1) / c.bn)) / cu;
}
TileChoice choose_tile(int64_t m, int64_t n, int64_t steps, hq_dtype out) {
    const float cu = static_cast<float>(hq::compute_units());
    TileChoice best{kTile64, 1e30f};
    for (const TileCost &c : kTiles) {
        const int o = out == HQ_F32;
        const float tiles = ceilf(tiles_per_cu(c, m, n, cu));
        const float us = c.begin + (tiles - 1.0f) * c.again + steps * std::max(c.round[o], tiles * c.each[o]);
        if (us < best.us) best = {c.tile, us};
    }
    return best;
}
TileChoice choose_pair(const ProductArgs &a, const ProductArgs &b, hq_dtype out) {
    const float cu = static_cast<float>(hq::compute_units());
    TileChoice best{kTile64, 1e30f};
    for (const TileCost &c : kTiles) {
        if (c.tile == kTile256) continue;
        const int o = out == HQ_F32;
        const float share = a.steps * tiles_per_cu(c, a.m, a.n, cu) * c.each[o] + b.steps * tiles_per_cu(c, b.m, b.n, cu) * c.each[1];
        // (the last round is only partly filled: half of the longer tile; charged where there is one round, too: 2048 x 960 -> 3840 is
        // estimated at 45.7 us for 184 workgroups of 256 x 128, 32.1 without it, and takes 64 x 128, 34.4)
        const float longest = std::max(a.steps * c.each[o], b.steps * c.each[1]);
        const float us = c.begin + std::max(std::max(a.steps * c.round[o], b.steps * c.round[1]), share + 0.5f * longest);
        if (us < best.us) best = {c.tile, us};
    }
    return best;
}

template <int OUT>
hq_status launch(const ProductArgs &a, Tile tile, hipStream_t st) {
    switch (tile) {
        case kTile256:
            // (not with fp32 results: too many registers)
            if constexpr (OUT != HQ_F32) return launch_tiles<OUT, 256, 256, 4, 2, 2>(a, st);
            [[fallthrough]];
        case kTile128: return launch_tiles<OUT, 256, 128, 4, 2, 3>(a, st);
        case kTile64x128: return launch_tiles<OUT, 64, 128, 2, 2, 3>(a, st);
        default: return launch_tiles<OUT, 64, 64, 2, 2, 3>(a, st);
    }
}

template <int OUT>
hq_status launch_pair(const ProductArgs &a, const ProductArgs &b, const hq::Fp8Sums &sums, Tile tile, hipStream_t st) {
    switch (tile) {
        case kTile128: return launch_pair<OUT, 256, 128, 4, 2, 3>(a, b, sums, st);
        case kTile64x128: return launch_pair<OUT, 64, 128, 2, 2, 3>(a, b, sums, st);
        default: return launch_pair<OUT, 64, 64, 2, 2, 3>(a, b, sums, st);
    }
}

ProductArgs product_args(const uint8_t *xq, const float *x_scale, const uint8_t *wq, const float *w_scale, bool scale_turned,
                         const void *bias, int64_t m, int n, int k, void *y) {
    const int steps = static_cast<int>(hq::fp8_groups(k)), blocks = static_cast<int>(hq::fp8_groups(n));
    return {xq, wq, x_scale, w_scale, bias, y, m, n, hq::fp8_pitch(k), steps, scale_turned ? 1 : steps, scale_turned ? blocks : 1};
}

// What a product takes: a cut of K, or tiles.
struct ProductChoice {
    bool split;
    hq::Fp8Cut cut;
    TileChoice tile;
    float us() const { return split ? cut.us : tile.us; }
};
ProductChoice choose(int64_t m, int64_t n, int64_t steps, hq_dtype out) {
    const hq::Fp8Cut cut = hq::fp8_split_cut(m, n, steps, nullptr, out);
    const TileChoice tile = choose_tile(m, n, steps, out);
    return {cut.us < tile.us, cut, tile};
}

hq_status product(const ProductArgs &a, hq_dtype dt, hipStream_t st) {
    const ProductChoice c = choose(a.m, a.n, a.steps, dt);
    if (c.split) return hq::fp8_split(a, c.cut, nullptr, dt, 0, 0, dt, st);
    switch (dt) {
        case HQ_F16: return launch<HQ_F16>(a, c.tile.tile, st);
        case HQ_BF16: return launch<HQ_BF16>(a, c.tile.tile, st);
        default: return launch<HQ_F32>(a, c.tile.tile, st);
    }
}

// What two products take: one launch, with a cut of K or with tiles, or one launch each.
struct PairChoice {
    enum { kSplit, kTiles, kAlone } how;
    hq::Fp8Cut cut;
    Tile tile;
};
PairChoice choose_pair_launch(const ProductArgs &a, const ProductArgs &b, bool sums, hq_dtype dt) {
    const hq::Fp8Cut cut = hq::fp8_split_pair_cut(a, b, dt);
    const TileChoice tile = choose_pair(a, b, dt);
    const float alone = choose(a.m, a.n, a.steps, dt).us() + choose(b.m, b.n, b.steps, HQ_F32).us() + (sums ? 2.0f : 0.0f);
    const auto how = cut.us < tile.us && cut.us < alone ? PairChoice::kSplit : tile.us < alone ? PairChoice::kTiles : PairChoice::kAlone;
    return {how, cut, tile.tile};
}

// a with results of type dt, b with fp32 ones, and sums
hq_status product_pair(const ProductArgs &a, const ProductArgs &b, const hq::Fp8Sums &sums, hq_dtype dt, hipStream_t st) {
    const PairChoice c = choose_pair_launch(a, b, sums.parts != nullptr, dt);
    if (c.how == PairChoice::kSplit) return hq::fp8_split_pair(a, b, sums, c.cut, dt, st);
    if (c.how == PairChoice::kTiles) {
        switch (dt) {
            case HQ_F16: return launch_pair<HQ_F16>(a, b, sums, c.tile, st);
            case HQ_BF16: return launch_pair<HQ_BF16>(a, b, sums, c.tile, st);
            default: return launch_pair<HQ_F32>(a, b, sums, c.tile, st);
        }
    }
    if (sums.parts) {
        const hq::LaunchCheck check;
        sum_rows_kernel<<<sum_blocks(sums), 256, 0, st>>>(sums);
        if (const hq_status s = check.status()) return s;
    }
    if (const hq_status s = product(a, dt, st)) return s;
    return product(b, HQ_F32, st);
}

// Rows of codes whose tiles are addressed with 31-bit offsets, and tile counts that fit a grid (n is a size of 32 bits; m is bounded before
// it is multiplied).
bool product_fits(int64_t m, int64_t n, int64_t k) {
    return k <= (int64_t{1} << 31) / 256 - 16 && m <= int64_t{0x7FFFFFFF} * 16 && ((m + 15) / 16) * ((n + 15) / 16) <= 0x7FFFFFFF;
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
    return product(product_args(xq, x_scale, wq, w_scale, w_scale_turned != 0, bias, m, n, k, y), y_dtype,
                   static_cast<hipStream_t>(stream));
}

namespace {
// Whether a layer is one launch that quantises its rows as it multiplies (and with which cut), or two.
struct LayerChoice {
    bool one_launch;
    hq::Fp8Cut cut;
};
LayerChoice choose_layer(hq_dtype x_dtype, int64_t m, int n, int k, hq_dtype y_dtype) {
    const int64_t steps = hq::fp8_groups(k);
    const hq::Fp8Cut fused = hq::fp8_split_cut(m, n, steps, &x_dtype, y_dtype);
    // us of quantising them by themselves: 2.2 on the card, and a launch more on the host, which counts where calls follow one another
    // (16 x 4096 -> 4096: 6.8 against 8.4 us of one launch in a graph, called one by one 9.6 against 9.1)
    const float rows = 3.2f + static_cast<float>(m) * k * (hq::size_of(x_dtype) + 1) / 4.5e6f;
    return {fused.us < rows + choose(m, n, steps, y_dtype).us(), fused};
}
}  // namespace

extern "C" int64_t hq_act_quant_fp8_linear_workspace(hq_dtype x_dtype, int64_t m, int n, int k, hq_dtype y_dtype) {
    if (m <= 0 || n <= 0 || k <= 0 || choose_layer(x_dtype, m, n, k, y_dtype).one_launch) return 0;
    return up256(m * hq::fp8_pitch64(k)) + up256(4 * hq::fp8_groups(k) * m);
}

extern "C" hq_status hq_act_quant_fp8_linear(const void *x, hq_dtype x_dtype, int64_t row_stride, const uint8_t *wq, const float *w_scale,
                                             const void *bias, int64_t m, int n, int k, void *workspace, void *y, hq_dtype y_dtype,
                                             void *stream) {
    if (!wq || !w_scale || (m > 0 && (!x || !y))) return HQ_ERR_NULL;
    if (!hq::is_float(x_dtype) || !hq::is_float(y_dtype)) return HQ_ERR_DTYPE;
    if (m < 0 || n <= 0 || k <= 0 || row_stride < 0) return HQ_ERR_SHAPE;
    const int size = hq::size_of(y_dtype);
    if (!hq::aligned_to(x, hq::size_of(x_dtype)) || !hq::aligned16(wq) || !hq::aligned_to(w_scale, 4) || !hq::aligned16(workspace) ||
        !hq::aligned_to(y, size) || !hq::aligned_to(bias, size))
        return HQ_ERR_ALIGN;
    if (!product_fits(m, n, k) || !hq::fp8_fits(m, k)) return HQ_ERR_UNSUPPORTED;
    if (m == 0) return HQ_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ProductArgs p = product_args(nullptr, nullptr, wq, w_scale, false, bias, m, n, k, y);
    const LayerChoice choice = choose_layer(x_dtype, m, n, k, y_dtype);
    if (choice.one_launch) return hq::fp8_split(p, choice.cut, x, x_dtype, row_stride, k, y_dtype, st);
    if (!workspace) return HQ_ERR_NULL;
    uint8_t *xq = static_cast<uint8_t *>(workspace);
    float *sx = reinterpret_cast<float *>(xq + up256(m * hq::fp8_pitch64(k)));
    if (const hq_status s = hq::fp8_rows(x, x_dtype, m, k, row_stride, xq, sx, st)) return s;
    p.x = xq, p.sx = sx;
    return product(p, y_dtype, st);
}

namespace {
const char *name_of(const hq::Fp8Cut &c, bool one_launch) {
    if (one_launch)
        return c.nt == 1   ? "one launch (16 x 16)"
               : c.nt == 2 ? "one launch (16 x 32)"
               : c.nt == 4 ? "one launch (16 x 64)"
                           : "one launch (16 x 128)";
    return c.mt == 4 ? "split (64 x 64)" : c.mt == 2 ? "split (32 x 32)" : c.nt == 2 ? "split (16 x 32)" : "split (16 x 16)";
}
const char *name_of(Tile t) {
    switch (t) {
        case kTile256: return "tile (256 x 256)";
        case kTile128: return "tile (256 x 128)";
        case kTile64x128: return "tile (64 x 128)";
        default: return "tile (64 x 64)";
    }
}
}  // namespace

extern "C" const char *hq_fp8_linear_kernel_name(hq_dtype x_dtype, int64_t m, int n, int k, hq_dtype y_dtype) {
    if (m <= 0 || n <= 0 || k <= 0 || !hq::is_float(y_dtype) || !product_fits(m, n, k)) return "none";
    if (hq::is_float(x_dtype)) {
        const LayerChoice l = choose_layer(x_dtype, m, n, k, y_dtype);
        if (l.one_launch) return name_of(l.cut, true);
    }
    const ProductChoice c = choose(m, n, hq::fp8_groups(k), y_dtype);
    return c.split ? name_of(c.cut, false) : name_of(c.tile.tile);
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
    if (!product_fits(m, k, n) || !product_fits(n, k, m) || !hq::fp8_fits(m, n) || !hq::fp8_fits(m, k) ||
        hq::fp8_groups(m) * (hq::fp8_groups(n) + hq::fp8_groups(k)) > 0x7FFFFFFF)
        return HQ_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (m == 0) {
        const hq::LaunchCheck check;
        const int64_t count = static_cast<int64_t>(n) * k;
        zero_kernel<<<static_cast<uint32_t>(std::min<int64_t>(1024, (count + 255) / 256)), 256, 0, st>>>(dw, count);
        if (db) zero_kernel<<<std::min<uint32_t>(1024, (n + 255) / 256), 256, 0, st>>>(db, n);
        return check.status();
    }
    uint8_t *base = static_cast<uint8_t *>(workspace);
    const BackwardSpace at(m, n, k);
    const auto f32 = [&](int64_t offset) { return reinterpret_cast<float *>(base + offset); };
    const hq::Fp8Gradient q{base + at.dyq, base + at.dyq_t, base + at.xq_t, f32(at.dy_scale), f32(at.dy_scale_t), f32(at.x_scale),
                            db ? f32(at.sums) : nullptr};
    if (const hq_status s = hq::fp8_gradient(dy, dy_stride, x, x_stride, dtype, m, n, k, q, st)) return s;
    // dx [m, k] = dy [m, n] W [n, k]: the weights' codes with rows of n, their scales as those of W
    const ProductArgs for_x = product_args(q.dyq, q.dy_scale, wq_t, w_scale, true, nullptr, m, k, n, dx);
    // dW [n, k] = dy^T [n, m] x [m, k]
    const ProductArgs for_w = product_args(q.dyq_t, q.dy_scale_t, q.xq_t, q.x_scale, true, nullptr, n, k, static_cast<int>(m), dw);
    return product_pair(for_x, for_w, {q.sums, hq::fp8_groups(m), n, db}, dtype, st);
}

extern "C" const char *hq_fp8_linear_backward_kernel_name(hq_dtype dtype, int64_t m, int n, int k, int bias_grad) {
    if (m <= 0 || n <= 0 || k <= 0 || !hq::is_float(dtype) || !product_fits(m, k, n) || !product_fits(n, k, m)) return "none";
    const ProductArgs x = product_args(nullptr, nullptr, nullptr, nullptr, true, nullptr, m, k, n, nullptr);
    const ProductArgs w = product_args(nullptr, nullptr, nullptr, nullptr, true, nullptr, n, k, static_cast<int>(m), nullptr);
    const PairChoice c = choose_pair_launch(x, w, bias_grad != 0, dtype);
    return c.how == PairChoice::kSplit ? name_of(c.cut, false) : c.how == PairChoice::kTiles ? name_of(c.tile) : "two launches";
}
