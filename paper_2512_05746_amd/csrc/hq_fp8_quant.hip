// Quantisers of 8-bit floats (E4M3: 4 bits of exponent, 3 of mantissa, largest value 448) with a scale for each tile of values:
// 128 neighbours of a row, 128 neighbours of a column, or a block of 128 x 128.
//
//     amax = max |x| over the tile;  s = 1 if amax is 0, else max(amax * c, 2^-126);  code = E4M3(x * (1 / s))
//
// c is 1/448 in fp32, and products and quotient are rounded to nearest, so that the codes are a function of the inputs alone; the
// conversion rounds to nearest, ties to even.  |x (1 / s)| is at most 448 (1 + 2^-22), which rounds to 448.  A tile that holds an
// infinity or a NaN gets a NaN for its scale and zeros for codes: every product that uses it is NaN.
//
// Bound by memory: a value is read once and written as one byte, or as two bytes where codes along rows and along columns are wanted.
// rows_kernel: 16 lanes own 128 values of a row, 8 each; 8192 x 4096 in bf16 20.5 us (4.9 TB/s).
// tile: a workgroup of 256 threads owns a tile of 128 x 128; a thread holds 8 rows x 8 columns as they came from memory, so a maximum
// along a row is one over 16 lanes, along a column one over 16 threads at the same columns (4 lanes of each wave, then LDS), and the
// codes of a column leave through LDS as whole pieces of 128 bytes.  Values of 16 bits are compared two at a time by their bits; the
// scales of a wave's 8 rows are taken in 8 lanes at once (a division each), not in every lane for every row; tiles that lie inside have
// no bounds to check: together 79 -> 41 us for the gradient and the activations of 8192 x (4096 + 4096) in bf16 (224 MB, 5.4 TB/s), 15.6
// -> 9.7 for 2048 x (3840 + 960) in fp16.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hq_common.h"
#include "hq_floats.h"
#include "hq_fp8.h"
#include "hq_fp8_codes.h"

namespace {

struct RowsArgs {
    const void *x;
    int64_t m, row_stride;
    int k, pitch;          // values and bytes of codes a row
    uint8_t *xq;           // [m, pitch]
    float *scale;          // [k / 128, m]
};

template <int DT>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
    using T = typename Float<DT>::type;
    const int lane16 = threadIdx.x & 15;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
    if (row >= a.m) return;
    const int groups = (a.k + kGroup - 1) / kGroup;
    const T *x = static_cast<const T *>(a.x) + row * a.row_stride;
    for (int b = blockIdx.y; b < groups; b += gridDim.y) {
        const int c = b * kGroup + lane16 * 8;
        Raw8<T> raw;
        if (c + 8 <= a.k) raw.load(x + c);
        else raw.load_some(x + c, a.k - c);
        Tops<T> top;
        top.add(raw);
        float v[8];
        raw.floats(v);
        const float s = scale_of(max_lanes<16>(top.all())), inverse = inverse_of(s);
        if (c < a.pitch) *reinterpret_cast<uint2 *>(a.xq + row * a.pitch + c) = uint2{codes4(v, inverse), codes4(v + 4, inverse)};
        if (lane16 == 0) a.scale[static_cast<int64_t>(b) * a.m + row] = s;
    }
}

struct TileArgs {
    const void *x;          // [rows, columns]
    int64_t rows, row_stride;
    int columns;
    int pitch;              // bytes a row of q
    int64_t pitch_t;        // bytes a row of q_t
    uint8_t *q;             // [rows, pitch], or null
    uint8_t *q_t;           // [columns, pitch_t], or null
    float *scale;           // of rows: [columns / 128, rows]; of blocks: [rows / 128, columns / 128]
    float *scale_t;         // of columns: [rows / 128, columns]
    float *sums;            // [rows / 128, columns]: sums of a tile's columns; or null
};

struct TileSpace {
    __attribute__((aligned(16))) uint8_t turned[kGroup * kGroup];
    uint32_t top_of[4][kGroup];
    float sum_of[4][kGroup], inverse_t[kGroup];
};

// the value of lane N of each row of 16 lanes
template <int N>
__device__ __forceinline__ float of_lane(float v) {
    return __int_as_float(dpp<0x150 + N>(__float_as_int(v)));
}

// Tile (bx, by).  BLOCKS: one scale for the tile; otherwise codes along the rows in q and along the columns in q_t.  WHOLE: it lies inside.
template <int DT, bool BLOCKS, bool WHOLE>
__device__ __forceinline__ void tile_body(const TileArgs &a, TileSpace &lds, uint32_t bx, uint32_t by) {
    using T = typename Float<DT>::type;
    const int tid = threadIdx.x, lane16 = tid & 15, part = tid >> 4, wave = tid >> 6;
    const int64_t row0 = static_cast<int64_t>(by) * kGroup, my_row = row0 + part * 8;
    const int column0 = bx * kGroup, c = column0 + lane16 * 8;
    const int blocks_across = (a.columns + kGroup - 1) / kGroup;

    Raw8<T> raw[8];   // of 8 rows
    Tops<T> tops;     // of the columns
    {
        const T *from = static_cast<const T *>(a.x) + my_row * a.row_stride + c;
#pragma unroll
        for (int r = 0; r < 8; ++r, from += a.row_stride) {
            if (WHOLE || (my_row + r < a.rows && c + 8 <= a.columns)) raw[r].load(from);
            else if (my_row + r < a.rows && c < a.columns) raw[r].load_some(from, a.columns - c);
            else raw[r].zero();
        }
    }
    float inverse[8];   // of the rows
    if constexpr (BLOCKS) {
#pragma unroll
        for (int r = 0; r < 8; ++r) tops.add(raw[r]);
        const uint32_t t = max_lanes<64>(tops.all());
        if ((tid & 63) == 0) lds.top_of[wave][0] = t;
        __syncthreads();
        const float s = scale_of(max(max(lds.top_of[0][0], lds.top_of[1][0]), max(lds.top_of[2][0], lds.top_of[3][0])));
        const float inv = inverse_of(s);
#pragma unroll
        for (int r = 0; r < 8; ++r) inverse[r] = inv;
        if (tid == 0) a.scale[static_cast<int64_t>(by) * blocks_across + bx] = s;
    } else {
        // Rows: lane r of 16 gets the maximum of row r, takes its scale, and hands the inverse to the others.
        uint32_t mine = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            Tops<T> row;
            row.add(raw[r]);
            const uint32_t t = max_lanes<16>(row.all());
            mine = lane16 == r ? t : mine;
            tops.add(raw[r]);
        }
        const float s_row = scale_of(mine), inv = inverse_of(s_row);
        inverse[0] = of_lane<0>(inv), inverse[1] = of_lane<1>(inv), inverse[2] = of_lane<2>(inv), inverse[3] = of_lane<3>(inv);
        inverse[4] = of_lane<4>(inv), inverse[5] = of_lane<5>(inv), inverse[6] = of_lane<6>(inv), inverse[7] = of_lane<7>(inv);
        if (lane16 < 8 && (WHOLE || my_row + lane16 < a.rows)) a.scale[static_cast<int64_t>(bx) * a.rows + my_row + lane16] = s_row;
        // columns: over the 4 lanes of a wave that share them, then over the waves
        tops.join([](int v) { return __shfl_xor(v, 16); });
        tops.join([](int v) { return __shfl_xor(v, 32); });
        float sum[8];
        if (a.sums) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[i] = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) sum[i] += static_cast<float>(raw[r].v[i]);
                sum[i] += __shfl_xor(sum[i], 16);
                sum[i] += __shfl_xor(sum[i], 32);
            }
        }
        if ((tid & 63) < 16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lds.top_of[wave][lane16 * 8 + i] = tops.column(i);
                if (a.sums) lds.sum_of[wave][lane16 * 8 + i] = sum[i];
            }
        }
        __syncthreads();
        if (tid < kGroup) {
            const float s = scale_of(max(max(lds.top_of[0][tid], lds.top_of[1][tid]), max(lds.top_of[2][tid], lds.top_of[3][tid])));
            lds.inverse_t[tid] = inverse_of(s);
            if (WHOLE || column0 + tid < a.columns) {
                const int64_t at = static_cast<int64_t>(by) * a.columns + column0 + tid;
                a.scale_t[at] = s;
                if (a.sums) a.sums[at] = (lds.sum_of[0][tid] + lds.sum_of[1][tid]) + (lds.sum_of[2][tid] + lds.sum_of[3][tid]);
            }
        }
        __syncthreads();
    }

    // codes along the rows
    if (a.q) {
        uint8_t *to = a.q + my_row * a.pitch + c;
#pragma unroll
        for (int r = 0; r < 8; ++r, to += a.pitch) {
            float v[8];
            raw[r].floats(v);
            if (WHOLE || (my_row + r < a.rows && c < a.pitch))
                *reinterpret_cast<uint2 *>(to) = uint2{codes4(v, inverse[r]), codes4(v + 4, inverse[r])};
        }
    }
    if (!a.q_t) return;

    // Codes along the columns: a thread's 8 rows of a column are 8 bytes of that column's 128.  The 8-byte pieces of a column are
    // kept in an order that depends on column / 8, so that 16 lanes write to different banks.
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int column = lane16 * 8 + i;
        const float inv = BLOCKS ? inverse[0] : lds.inverse_t[column];
        float t[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) t[r] = static_cast<float>(raw[r].v[i]);
        *reinterpret_cast<uint2 *>(lds.turned + column * kGroup + ((part ^ lane16) * 8)) = uint2{codes4(t, inv), codes4(t + 4, inv)};
    }
    __syncthreads();
    uint8_t *to = a.q_t + static_cast<int64_t>(column0 + part) * a.pitch_t + row0 + lane16 * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i, to += 16 * a.pitch_t) {
        const int column = i * 16 + part;
        if (WHOLE || (column0 + column < a.columns && row0 + lane16 * 8 < a.pitch_t))
            *reinterpret_cast<uint2 *>(to) =
                *reinterpret_cast<const uint2 *>(lds.turned + column * kGroup + ((lane16 ^ (column >> 3)) * 8));
    }
}
template <int DT, bool BLOCKS>
__device__ __forceinline__ void tile(const TileArgs &a, TileSpace &lds, uint32_t bx, uint32_t by) {
    if ((by + 1) * static_cast<int64_t>(kGroup) <= a.rows && static_cast<int64_t>(bx + 1) * kGroup <= a.columns)
        tile_body<DT, BLOCKS, true>(a, lds, bx, by);
    else
        tile_body<DT, BLOCKS, false>(a, lds, bx, by);
}

template <int DT>
__global__ __launch_bounds__(256) void blocks_kernel(TileArgs a) {
    __shared__ TileSpace lds;
    tile<DT, true>(a, lds, blockIdx.x, blockIdx.y);
}

// A gradient, both ways, and the activations, in blocks: what a backward pass quantises, in one launch.  across: tiles in a row of each;
// the first `first` workgroups are the gradient's.
template <int DT>
__global__ __launch_bounds__(256) void gradient_kernel(TileArgs dy, TileArgs x, uint32_t dy_across, uint32_t x_across, uint32_t first) {
    __shared__ TileSpace lds;
    if (blockIdx.x < first) tile<DT, false>(dy, lds, blockIdx.x % dy_across, blockIdx.x / dy_across);
    else tile<DT, true>(x, lds, (blockIdx.x - first) % x_across, (blockIdx.x - first) / x_across);
}

template <class F>
hq_status for_dtype(hq_dtype dt, F f) {
    switch (dt) {
        case HQ_F16: return f(std::integral_constant<int, HQ_F16>{});
        case HQ_BF16: return f(std::integral_constant<int, HQ_BF16>{});
        case HQ_F32: return f(std::integral_constant<int, HQ_F32>{});
        default: return HQ_ERR_DTYPE;
    }
}

}  // namespace

namespace hq {

hq_status fp8_rows(const void *x, hq_dtype dt, int64_t m, int k, int64_t row_stride, uint8_t *xq, float *scale, hipStream_t st) {
    const RowsArgs a{x, m, row_stride, k, fp8_pitch(k), xq, scale};
    const int groups = (k + kGroup - 1) / kGroup;
    const uint32_t bx = static_cast<uint32_t>((m + 15) / 16);
    // few rows: a workgroup for each group of 128; many: a workgroup keeps its rows, up to about 16 workgroups a CU
    const uint32_t want = std::max<uint32_t>(1, static_cast<uint32_t>(compute_units()) * 16 / bx);
    const dim3 grid(bx, std::min<uint32_t>(groups, want));
    return for_dtype(dt, [&](auto d) {
        const LaunchCheck check;
        rows_kernel<decltype(d)::value><<<grid, 256, 0, st>>>(a);
        return check.status();
    });
}

hq_status fp8_blocks(const void *x, hq_dtype dt, int64_t rows, int columns, int64_t row_stride, uint8_t *q, uint8_t *q_t, float *scale,
                     hipStream_t st) {
    const TileArgs a{x, rows, row_stride, columns, fp8_pitch(columns), fp8_pitch64(rows), q, q_t, scale, nullptr, nullptr};
    const dim3 grid((columns + kGroup - 1) / kGroup, static_cast<uint32_t>((rows + kGroup - 1) / kGroup));
    return for_dtype(dt, [&](auto d) {
        const LaunchCheck check;
        blocks_kernel<decltype(d)::value><<<grid, 256, 0, st>>>(a);
        return check.status();
    });
}

hq_status fp8_gradient(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, hq_dtype dt, int64_t m, int n, int k,
                       const Fp8Gradient &out, hipStream_t st) {
    const TileArgs g{dy, m, dy_stride, n, fp8_pitch(n), fp8_pitch64(m), out.dyq, out.dyq_t, out.dy_scale, out.dy_scale_t, out.sums};
    const TileArgs b{x, m, x_stride, k, fp8_pitch(k), fp8_pitch64(m), nullptr, out.xq_t, out.x_scale, nullptr, nullptr};
    const int64_t down = fp8_groups(m), dy_across = fp8_groups(n), x_across = fp8_groups(k);
    return for_dtype(dt, [&](auto d) {
        const LaunchCheck check;
        gradient_kernel<decltype(d)::value><<<static_cast<uint32_t>(down * (dy_across + x_across)), 256, 0, st>>>(
            g, b, static_cast<uint32_t>(dy_across), static_cast<uint32_t>(x_across), static_cast<uint32_t>(down * dy_across));
        return check.status();
    });
}

}  // namespace hq

extern "C" hq_status hq_fp8_quantize_rows(const void *x, hq_dtype x_dtype, int64_t m, int k, int64_t row_stride, uint8_t *xq,
                                          float *x_scale, void *stream) {
    if (m > 0 && (!x || !xq || !x_scale)) return HQ_ERR_NULL;
    if (!hq::is_float(x_dtype)) return HQ_ERR_DTYPE;
    if (m < 0 || k <= 0 || row_stride < 0) return HQ_ERR_SHAPE;
    if (!hq::aligned_to(x, hq::size_of(x_dtype)) || !hq::aligned16(xq) || !hq::aligned_to(x_scale, 4)) return HQ_ERR_ALIGN;
    if (!hq::fp8_fits(m, k)) return HQ_ERR_UNSUPPORTED;
    if (m == 0) return HQ_OK;
    return hq::fp8_rows(x, x_dtype, m, k, row_stride, xq, x_scale, static_cast<hipStream_t>(stream));
}

extern "C" hq_status hq_fp8_quantize_blocks(const void *w, hq_dtype w_dtype, int64_t n, int k, int64_t row_stride, uint8_t *wq,
                                            uint8_t *wq_t, float *w_scale, void *stream) {
    if (!w || (!wq && !wq_t) || !w_scale) return HQ_ERR_NULL;
    if (!hq::is_float(w_dtype)) return HQ_ERR_DTYPE;
    if (n <= 0 || k <= 0 || row_stride < 0) return HQ_ERR_SHAPE;
    if (!hq::aligned_to(w, hq::size_of(w_dtype)) || !hq::aligned16(wq) || !hq::aligned16(wq_t) || !hq::aligned_to(w_scale, 4))
        return HQ_ERR_ALIGN;
    if (!hq::fp8_fits(n, k)) return HQ_ERR_UNSUPPORTED;
    return hq::fp8_blocks(w, w_dtype, n, k, row_stride, wq, wq_t, w_scale, static_cast<hipStream_t>(stream));
}
