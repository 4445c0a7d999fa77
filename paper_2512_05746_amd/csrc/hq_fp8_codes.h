// Scales and E4M3 codes of values in registers (the definition is in hq_fp8_quant.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_floats.h"
#include "hq_fp8.h"

namespace {

constexpr int kGroup = hq::kFp8Group;

__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float s = fmaxf(__uint_as_float(amax_bits) * (1.0f / 448.0f), 0x1p-126f);
    return amax_bits == 0 ? 1.0f : s;
}
// (0 for a tile that is not finite: its codes are taken from zeros)
__device__ __forceinline__ float inverse_of(float s) { return s == s ? __fdiv_rn(1.0f, s) : 0.0f; }

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// codes of 4 values in a dword; `inverse` is 0 for a tile that is not finite
__device__ __forceinline__ uint32_t codes4(const float *v, float inverse) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, w, true);
    return inverse == 0.0f ? 0u : static_cast<uint32_t>(w);
}

// 8 neighbouring values as they are in memory
template <class T> struct Raw8 {
    typename Vec<T, 8>::type v;
    __device__ __forceinline__ void load(const T *from) { v = load_vec<T, 8>(from); }
    // those below `count` (of 8); zeros for the others
    __device__ __forceinline__ void load_some(const T *from, int count) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? from[i] : static_cast<T>(0.0f);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(0.0f);
    }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(v[i]);
    }
};

// The largest magnitudes of values by their bits, of each of 8 columns: floats of 16 bits two at a time.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <class T> struct Tops {
    u16x2 t[4] = {};
    __device__ __forceinline__ void add(const Raw8<T> &r) {
        const u32x4 w = __builtin_bit_cast(u32x4, r.v) & 0x7FFF7FFFu;
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = __builtin_elementwise_max(t[i], __builtin_bit_cast(u16x2, static_cast<uint32_t>(w[i])));
    }
    // with the values of the lane that `from` names
    template <class F> __device__ __forceinline__ void join(F from) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            t[i] = __builtin_elementwise_max(t[i], __builtin_bit_cast(u16x2, from(__builtin_bit_cast(int, t[i]))));
    }
    // as the bits of a float
    __device__ __forceinline__ static uint32_t wide(unsigned short bits) {
        return __float_as_uint(static_cast<float>(__builtin_bit_cast(T, bits)));
    }
    __device__ __forceinline__ uint32_t column(int i) const { return wide(t[i / 2][i & 1]); }
    __device__ __forceinline__ uint32_t all() const {
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(t[0], t[1]), __builtin_elementwise_max(t[2], t[3]));
        return wide(m[0] > m[1] ? m[0] : m[1]);
    }
};
template <> struct Tops<float> {
    uint32_t t[8] = {};
    __device__ __forceinline__ void add(const Raw8<float> &r) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = max(t[i], magnitude(r.v[i]));
    }
    template <class F> __device__ __forceinline__ void join(F from) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = max(t[i], static_cast<uint32_t>(from(static_cast<int>(t[i]))));
    }
    __device__ __forceinline__ uint32_t column(int i) const { return t[i]; }
    __device__ __forceinline__ uint32_t all() const {
        return max(max(max(t[0], t[1]), max(t[2], t[3])), max(max(t[4], t[5]), max(t[6], t[7])));
    }
};

}  // namespace
