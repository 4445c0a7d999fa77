// Heads dealt to lanes, 8 neighbouring channels each: the Hadamard transform, 4-bit codes, and the numbers they stand for.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_floats.h"

namespace {

// Which 8 channels of a head a lane has: block number kv4_block(in), so that blocks whose numbers differ in one bit are in lanes that one
// permute exchanges: bits 0 and 1 inside quads, bit 2 in a mirrored half row (lane i ^ 7), bit 3 in a mirrored row (i ^ 15).  Heads begin at a
// lane that is a multiple of their lanes, a power of two.
__host__ __device__ __forceinline__ int kv4_block(int in) { return (in & 19) ^ (in & 4 ? 7 : 0) ^ (in & 8 ? 12 : 0); }

// sum[i] += factor[i] * x[i] of the lane whose block differs in bit BIT, rounded once.  One instruction each, which the compiler does not form
// by itself from a permute and a multiply-add (there is none with three addresses).  A permute reads a register at the earliest two
// instructions after it was written.
#define HQ_LANES(i, ctrl) "v_fmac_f32_dpp %" #i ", %[x" #i "], %[f" #i "] " ctrl " row_mask:0xf bank_mask:0xf\n\t"
#define HQ_LANES8(ctrl)                                                                                                                    \
    asm("s_nop 1\n\t" HQ_LANES(0, ctrl) HQ_LANES(1, ctrl) HQ_LANES(2, ctrl) HQ_LANES(3, ctrl) HQ_LANES(4, ctrl) HQ_LANES(5, ctrl)           \
            HQ_LANES(6, ctrl) HQ_LANES(7, ctrl)                                                                                           \
        : "+&v"(sum[0]), "+&v"(sum[1]), "+&v"(sum[2]), "+&v"(sum[3]), "+&v"(sum[4]), "+&v"(sum[5]), "+&v"(sum[6]), "+&v"(sum[7])                  \
        : [x0] "v"(x[0]), [x1] "v"(x[1]), [x2] "v"(x[2]), [x3] "v"(x[3]), [x4] "v"(x[4]), [x5] "v"(x[5]), [x6] "v"(x[6]), [x7] "v"(x[7]),   \
          [f0] "v"(f[0]), [f1] "v"(f[1]), [f2] "v"(f[2]), [f3] "v"(f[3]), [f4] "v"(f[4]), [f5] "v"(f[5]), [f6] "v"(f[6]), [f7] "v"(f[7]))
template <int BIT>
__device__ __forceinline__ void add_lanes(float (&sum)[8], const float (&x)[8], const float (&f)[8]) {
    if constexpr (BIT == 0) HQ_LANES8("quad_perm:[1,0,3,2]");
    else if constexpr (BIT == 1) HQ_LANES8("quad_perm:[2,3,0,1]");
    else if constexpr (BIT == 2) HQ_LANES8("row_half_mirror");
    else HQ_LANES8("row_mirror");
}
#undef HQ_LANES8
#undef HQ_LANES
// One step between lanes: sums in the lanes whose bit is 0, differences in the others, which come with the opposite sign: own value minus
// the other lane's (a multiply-add by 1 or -1 into the value itself: 8 instructions instead of 16).
#define HQ_STEP(i, ctrl) "v_fmac_f32_dpp %" #i ", %" #i ", %8 " ctrl " row_mask:0xf bank_mask:0xf\n\t"
#define HQ_STEP8(ctrl)                                                                                                                     \
    asm("s_nop 1\n\t" HQ_STEP(0, ctrl) HQ_STEP(1, ctrl) HQ_STEP(2, ctrl) HQ_STEP(3, ctrl) HQ_STEP(4, ctrl) HQ_STEP(5, ctrl) HQ_STEP(6, ctrl) \
            HQ_STEP(7, ctrl)                                                                                                              \
        : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7])                                       \
        : "v"(sign))
template <int BIT>
__device__ __forceinline__ void walsh_lanes(float (&v)[8], int block) {
    const float sign = block >> BIT & 1 ? -1.0f : 1.0f;
    if constexpr (BIT == 0) HQ_STEP8("quad_perm:[1,0,3,2]");
    else if constexpr (BIT == 1) HQ_STEP8("quad_perm:[2,3,0,1]");
    else if constexpr (BIT == 2) HQ_STEP8("row_half_mirror");
    else HQ_STEP8("row_mirror");
}
#undef HQ_STEP8
#undef HQ_STEP
template <int STEP>
__device__ __forceinline__ void walsh_own(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(i & STEP)) {
            const float a = v[i], b = v[i + STEP];
            v[i] = a + b;
            v[i + STEP] = a - b;
        }
}
// The transform of blocks of 2^log2 channels (up to 128: 16 lanes), without its factor, walsh_factor; `block`: the lane's 8 channels.
__device__ __forceinline__ void walsh(float (&v)[8], int block, int log2) {
    if (log2 > 0) walsh_own<1>(v);
    if (log2 > 1) walsh_own<2>(v);
    if (log2 > 2) walsh_own<4>(v);
    if (log2 > 3) walsh_lanes<0>(v, block);
    if (log2 > 4) walsh_lanes<1>(v, block);
    if (log2 > 5) walsh_lanes<2>(v, block);
    if (log2 > 6) walsh_lanes<3>(v, block);
}
// The same for heads of LP lanes; blocks of all their channels (or 128) without a branch between the steps, which would move all values.
template <int LP>
__device__ __forceinline__ void walsh_of(float (&v)[8], int block, int log2) {
    constexpr int FULL = LP == 4 ? 5 : LP == 8 ? 6 : 7;
    if (log2 == FULL) {
        walsh_own<1>(v);
        walsh_own<2>(v);
        walsh_own<4>(v);
        walsh_lanes<0>(v, block);
        walsh_lanes<1>(v, block);
        if constexpr (FULL > 5) walsh_lanes<2>(v, block);
        if constexpr (FULL > 6) walsh_lanes<3>(v, block);
    } else {
        walsh(v, block, log2);
    }
}
// 2^(-log2 / 2) and the sign that the steps between lanes left the lane with.
__device__ __forceinline__ float walsh_factor(int block, int log2) {
    const float f = __builtin_ldexpf(log2 & 1 ? 0.70710678118654752f : 1.0f, -(log2 >> 1));
    const int bits = log2 > 3 ? block & ((1 << (log2 - 3)) - 1) : 0;
    return __builtin_popcount(bits) & 1 ? -f : f;
}

// ---- codes ------------------------------------------------------------------------------------------------------------
// The scale of a head from its largest magnitude: NaN where that is not finite (the codes are then 0).  A sixth to the nearest: the rounded
// product's remainder is exact, and so is its sixth's part in the second product.
__device__ __forceinline__ float kv4_scale(float top) {
    constexpr float SIXTH = 1.0f / 6.0f;
    const float q = top * SIXTH, scale = fmaxf(fmaf(fmaf(-6.0f, q, top), SIXTH, q), 0x1p-126f);
    return top == 0.0f ? 1.0f : top < __builtin_inff() ? scale : __builtin_nanf("");
}
// E2M1 codes of 8 numbers, to nearest, ties to even, the first in the low bits.
__device__ __forceinline__ uint32_t kv4_codes(const float (&t)[8]) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[0], t[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[2], t[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[4], t[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[6], t[7], 1.0f, 3);
    return w;
}
// Of the lane whose block differs in bit BIT.
template <int BIT>
__device__ __forceinline__ double of_lane_wide(double v) {
    constexpr int CTRL = BIT == 0 ? 0xB1 : BIT == 1 ? 0x4E : BIT == 2 ? 0x141 : 0x140;
    return __hiloint2double(dpp<CTRL>(__double2hiint(v)), dpp<CTRL>(__double2loint(v)));
}
template <int BIT>
__device__ __forceinline__ void other_lanes_wide(const double (&v)[8], double (&to)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = of_lane_wide<BIT>(v[i]);
}
template <int BIT>
__device__ __forceinline__ void walsh_lanes_wide(double (&v)[8], int block) {
    const double sign = block >> BIT & 1 ? -1.0 : 1.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = of_lane_wide<BIT>(v[i]) + sign * v[i];
}
// The transform in 64 bits, without its factor.
__device__ __forceinline__ void walsh_wide(double (&v)[8], int block, int log2) {
#pragma unroll
    for (int step = 1; step < 8; step *= 2)
        if (log2 > __builtin_ctz(step)) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(i & step)) {
                    const double a = v[i], b = v[i + step];
                    v[i] = a + b;
                    v[i + step] = a - b;
                }
        }
    if (log2 > 3) walsh_lanes_wide<0>(v, block);
    if (log2 > 4) walsh_lanes_wide<1>(v, block);
    if (log2 > 5) walsh_lanes_wide<2>(v, block);
    if (log2 > 6) walsh_lanes_wide<3>(v, block);
}
// Of LP lanes together: op by the steps of reduce_bits.
template <int LP, class Op>
__device__ __forceinline__ double reduce_wide(double v, Op op) {
    v = op(v, of_lane_wide<0>(v));
    v = op(v, of_lane_wide<1>(v));
    if constexpr (LP > 4) v = op(v, of_lane_wide<2>(v));
    if constexpr (LP > 8) v = op(v, of_lane_wide<3>(v));
    if constexpr (LP > 16) v = op(v, __shfl_xor(v, 16));
    return v;
}
// The codes of 8 of a head's sums, decided in 64 bits: 6 |sum| against each border times the largest of the head, ties to the even code.  Exact
// wherever the sums are (16-bit values whose sizes are within 2^30 of each other).  least: what the largest counts as at least (the scale has a
// least, 2^-126).
template <int LP>
__device__ __forceinline__ uint32_t kv4_codes_wide(const double (&sum)[8], double least) {
    double most = least;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmax(most, fabs(sum[i]));
    most = reduce_wide<LP>(most, [](double a, double b) { return fmax(a, b); });
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double x = 6.0 * fabs(sum[i]);
        uint32_t code = (x > 0.25 * most) + (x >= 0.75 * most) + (x > 1.25 * most) + (x >= 1.75 * most) + (x > 2.5 * most) +
                        (x >= 3.5 * most) + (x > 5.0 * most);
        if (sum[i] < 0.0) code |= 8;
        w |= code << (4 * i);
    }
    return w;
}

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
// The numbers of 8 codes, exact in 16 bits.
__device__ __forceinline__ half8v kv4_halves(uint32_t w) {
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The numbers of 8 codes as floats.
typedef float float2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void kv4_floats(uint32_t w, float (&v)[8]) {
    const float2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

template <class T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    constexpr int STEP = 16 / static_cast<int>(sizeof(T));
#pragma unroll
    for (int i = 0; i < 8; i += STEP) {
        const typename Vec<T, STEP>::type t = load_vec<T, STEP>(p + i);
#pragma unroll
        for (int e = 0; e < STEP; ++e) v[i + e] = static_cast<float>(t[e]);
    }
}
template <class T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    constexpr int STEP = 16 / static_cast<int>(sizeof(T));
#pragma unroll
    for (int i = 0; i < 8; i += STEP) {
        typename Vec<T, STEP>::type t;
#pragma unroll
        for (int e = 0; e < STEP; ++e) t[e] = round_to<T>(v[i + e]);
        store_vec<T, STEP>(p + i, t);
    }
}

}  // namespace
