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

// the value of the lane whose block differs in bit BIT
template <int BIT>
__device__ __forceinline__ float lane_of_bit(float v) {
    constexpr int CTRL = BIT == 0 ? 0xB1 : BIT == 1 ? 0x4E : BIT == 2 ? 0x141 : 0x140;
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// One step between lanes: sums in the lanes whose bit is 0, differences in the others.
template <int BIT>
__device__ __forceinline__ void walsh_lanes(float (&v)[8], int block) {
    const float sign = block >> BIT & 1 ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = lane_of_bit<BIT>(v[i]) + v[i] * sign;   // (the product is exact)
}
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
// The transform of blocks of 2^log2 channels (up to 128: 16 lanes), without its factor 2^(-log2 / 2); `block`: the lane's 8 channels.
__device__ __forceinline__ void walsh(float (&v)[8], int block, int log2) {
    if (log2 > 0) walsh_own<1>(v);
    if (log2 > 1) walsh_own<2>(v);
    if (log2 > 2) walsh_own<4>(v);
    if (log2 > 3) walsh_lanes<0>(v, block);
    if (log2 > 4) walsh_lanes<1>(v, block);
    if (log2 > 5) walsh_lanes<2>(v, block);
    if (log2 > 6) walsh_lanes<3>(v, block);
}
__device__ __forceinline__ float walsh_factor(int log2) {
    return __builtin_ldexpf(log2 & 1 ? 0.70710678118654752f : 1.0f, -(log2 >> 1));
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
