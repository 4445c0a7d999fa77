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
// 2^(-log2 / 2) and the sign that the steps between lanes left the lane with.
__device__ __forceinline__ float walsh_factor(int block, int log2) {
    const float f = __builtin_ldexpf(log2 & 1 ? 0.70710678118654752f : 1.0f, -(log2 >> 1));
    const int bits = log2 > 3 ? block & ((1 << (log2 - 3)) - 1) : 0;
    return __builtin_popcount(bits) & 1 ? -f : f;
}

// ---- codes ------------------------------------------------------------------------------------------------------------
// The scale of a head from the bits of its largest magnitude: NaN where that is not finite (the codes are then 0).
__device__ __forceinline__ float kv4_scale(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return amax_bits == 0 ? 1.0f : fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 6.0f), 0x1p-126f);
}
// E2M1 codes of 8 channels times `inverse` (0 for a head that is not finite), to nearest, ties to even, the first in the low bits
__device__ __forceinline__ uint32_t kv4_codes(const float (&v)[8], float inverse) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inverse, v[1] * inverse, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inverse, v[3] * inverse, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inverse, v[5] * inverse, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inverse, v[7] * inverse, 1.0f, 3);
    return inverse == 0.0f ? 0u : w;
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
