// 16- and 32-bit floats as arrays in memory: eight (or four) consecutive elements at a time, at any alignment of an element.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq.h"

namespace {

// element types by the numbers of hq_dtype
template <int DT> struct Float;
template <> struct Float<HQ_F16> { using type = _Float16; };
template <> struct Float<HQ_BF16> { using type = __bf16; };
template <> struct Float<HQ_F32> { using type = float; };

// Vectors in memory need the alignment of their elements only (the hardware takes wide accesses at any address).
template <class T, int N> struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
    typedef T memory __attribute__((ext_vector_type(N), aligned(alignof(T))));
};

template <class T, int N>
__device__ __forceinline__ typename Vec<T, N>::type load_vec(const T *p) {
    return *reinterpret_cast<const typename Vec<T, N>::memory *>(p);
}
template <class T, int N>
__device__ __forceinline__ void store_vec(T *p, const typename Vec<T, N>::type &v) {
    *reinterpret_cast<typename Vec<T, N>::memory *>(p) = v;
}

// (to nearest, ties to even: the conversion instructions)
template <class T>
__device__ __forceinline__ T round_to(float v) {
    return static_cast<T>(v);
}

// ---- reductions over neighbouring lanes -----------------------------------------------------------------------------
// Sums and maxima over groups of G lanes (a power of two), the same value in every lane.  The first four steps are lane
// permutes inside a row of 16 (once groups of 4 agree, a mirrored half row is an exchange of 4, a mirrored row one of 8).
template <int CTRL>
__device__ __forceinline__ int dpp(int v) {
    return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false);
}
template <int G, class Op>
__device__ __forceinline__ int reduce_bits(int v, Op op) {
    if constexpr (G > 1) v = op(v, dpp<0xB1>(v));    // quad permute 1 0 3 2
    if constexpr (G > 2) v = op(v, dpp<0x4E>(v));    // quad permute 2 3 0 1
    if constexpr (G > 4) v = op(v, dpp<0x141>(v));   // half row mirrored
    if constexpr (G > 8) v = op(v, dpp<0x140>(v));   // row mirrored
    if constexpr (G > 16) v = op(v, __shfl_xor(v, 16));
    if constexpr (G > 32) v = op(v, __shfl_xor(v, 32));
    return v;
}
template <int G>
__device__ __forceinline__ float sum_lanes(float v) {
    return __int_as_float(reduce_bits<G>(__float_as_int(v), [](int a, int b) {
        return __float_as_int(__int_as_float(a) + __int_as_float(b));
    }));
}
// of non-negative floats by their bits: a NaN is larger than any number
template <int G>
__device__ __forceinline__ uint32_t max_lanes(uint32_t v) {
    return static_cast<uint32_t>(reduce_bits<G>(static_cast<int>(v), [](int a, int b) {
        const uint32_t x = static_cast<uint32_t>(a), y = static_cast<uint32_t>(b);
        return static_cast<int>(x > y ? x : y);
    }));
}

}  // namespace
