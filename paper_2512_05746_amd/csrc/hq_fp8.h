// 8-bit floats with block scales: what the quantisers (hq_fp8_quant.hip) and the product (hq_fp8_linear.hip) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_common.h"

namespace hq {

constexpr int kFp8Group = 128;   // values that share a scale, along a row, a column, or both

// bytes of a row of codes: a multiple of 16, the end filled with zeros
inline int fp8_pitch(int values) { return (values + 15) & ~15; }
inline int64_t fp8_pitch64(int64_t values) { return (values + 15) & ~int64_t{15}; }
inline int64_t fp8_groups(int64_t values) { return (values + kFp8Group - 1) / kFp8Group; }

inline bool is_float(hq_dtype t) { return t == HQ_F16 || t == HQ_F32 || t == HQ_BF16; }
inline int size_of(hq_dtype t) { return t == HQ_F32 || t == HQ_I32 ? 4 : 2; }
inline bool aligned_to(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// sizes that the kernels index: a row of codes below 2 GiB, tiles of 128 rows below the grid's limit of 65535 in y
inline bool fp8_fits(int64_t rows, int64_t columns) {
    return columns <= 0x7FFFFF00 && rows <= int64_t{65535} * kFp8Group;
}

// The quantisers, without checks of their arguments.
hq_status fp8_rows(const void *x, hq_dtype dt, int64_t m, int k, int64_t row_stride, uint8_t *xq, float *scale, hipStream_t st);
hq_status fp8_blocks(const void *x, hq_dtype dt, int64_t rows, int columns, int64_t row_stride, uint8_t *q, uint8_t *q_t, float *scale,
                     hipStream_t st);
// What a backward pass quantises: dy [m, n] along its rows and along its columns, x [m, k] in blocks, transposed; the sums of 128 rows of
// dy.
struct Fp8Gradient {
    uint8_t *dyq, *dyq_t, *xq_t;              // [m, pitch of n], [n, pitch of m], [k, pitch of m]
    float *dy_scale, *dy_scale_t, *x_scale;   // [n / 128, m], [m / 128, n], [m / 128, k / 128]
    float *sums;                              // [m / 128, n], or null
};
hq_status fp8_gradient(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, hq_dtype dt, int64_t m, int n, int k,
                       const Fp8Gradient &out, hipStream_t st);

// A product's arguments.
struct Fp8Product {
    const uint8_t *x, *w;        // codes [m, pitch], [n, pitch]
    const float *sx, *sw;        // [steps, m]; sw[block of channels * sw_block + step * sw_step]
    const void *bias;            // [n] of the output type, or null
    void *y;                     // [m, n]
    int64_t m;
    int n, pitch, steps;
    int sw_block, sw_step;
};

// The product with K split over the waves of a workgroup (hq_fp8_split.hip): of codes, or of rows that it quantises itself.
struct Fp8Cut {
    int mt, nt;   // tiles of 16 tokens, of 16 channels, of a workgroup
    float us;     // estimated
};
// the best cut; in: the type of rows that are quantised, or null for codes
Fp8Cut fp8_split_cut(int64_t m, int64_t n, int64_t steps, const hq_dtype *in, hq_dtype out);
hq_status fp8_split(const Fp8Product &p, Fp8Cut cut, const void *x, hq_dtype x_dtype, int64_t row_stride, int k, hq_dtype out,
                    hipStream_t st);

// Two products in one launch, `a` with results of type out, `b` of fp32, and the sums over the rows of a matrix, both of a backward pass.
struct Fp8Sums {
    const float *parts;   // [rows, columns]; or null
    int64_t rows;
    int columns;
    float *out;           // [columns]
};
Fp8Cut fp8_split_pair_cut(const Fp8Product &a, const Fp8Product &b, hq_dtype out);
hq_status fp8_split_pair(const Fp8Product &a, const Fp8Product &b, const Fp8Sums &sums, Fp8Cut cut, hq_dtype out, hipStream_t st);

}  // namespace hq
