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
// codes along the rows and along the columns in one pass; sums (of the columns) may be null; sum_parts [rows / 128, columns]
hq_status fp8_both(const void *x, hq_dtype dt, int64_t rows, int columns, int64_t row_stride, uint8_t *q, float *scale, uint8_t *q_t,
                   float *scale_t, float *sum_parts, float *sums, hipStream_t st);

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
hq_status fp8_split(const Fp8Product &p, Fp8Cut cut, const void *x, hq_dtype x_dtype, int64_t row_stride, int k, hq_dtype out, hipStream_t st);

}  // namespace hq
