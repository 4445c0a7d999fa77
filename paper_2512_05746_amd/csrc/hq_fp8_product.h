// Product of E4M3 codes: arguments and matrix instructions, shared by its kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_buffer.h"
#include "hq_floats.h"
#include "hq_fp6.h"
#include "hq_fp8.h"

namespace {

constexpr int kStep = hq::kFp8Group;   // bytes of a row in one step, and values that share a scale

typedef float f32x4 __attribute__((ext_vector_type(4)));

using ProductArgs = hq::Fp8Product;

__device__ __forceinline__ f32x4 mfma_fp8(const v8i &a, const v8i &b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// Loads from memory straight into LDS.  They are written out: of the compiler's own it cannot tell which bytes they fill, and would let
// every read of LDS wait for all of them.  They have no register for a result.
__device__ __forceinline__ v4i words_of(const void *p, uint32_t bytes) {   // of a buffer's descriptor
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return v4i{static_cast<int>(at), static_cast<int>(at >> 32), static_cast<int>(bytes), 0x00027000};
}
// lane i's 16 (4) bytes to lds + 16 i (4 i); zeros from beyond the buffer
__device__ __forceinline__ void load16_to_lds(const v4i &buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "s"(lds) : "memory");
}
__device__ __forceinline__ void load4_to_lds(const v4i &buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "s"(lds) : "memory");
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct Halves {   // a lane's 32 codes of a step as operands of four bf16 instructions (E4M3 numbers are bf16 numbers)
    bf16x8 v[4];
};
__device__ __forceinline__ Halves halves_of(const v8i &codes) {
    Halves h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t w = static_cast<uint32_t>(codes[i]);
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
        const int at = (i & 1) * 4;
        h.v[i / 2][at] = a[0], h.v[i / 2][at + 1] = a[1], h.v[i / 2][at + 2] = b[0], h.v[i / 2][at + 3] = b[1];
    }
    return h;
}

// 16 columns of sums over the rows, by 256 threads: 16 to a column, each in the order of its rows; lds: 256 floats
__device__ __forceinline__ void sum_rows(const hq::Fp8Sums &s, uint32_t block, int tid, float *lds) {
    const int x = tid & 15, y = tid >> 4, c = block * 16 + x;
    float t = 0.0f;
    if (tid < 256 && c < s.columns)
        for (int64_t r = y; r < s.rows; r += 16) t += s.parts[r * s.columns + c];
    if (tid < 256) lds[y * 16 + x] = t;
    __syncthreads();
    if (tid < 16 && c < s.columns) {
#pragma unroll
        for (int i = 1; i < 16; ++i) t += lds[i * 16 + x];
        s.out[c] = t;
    }
}
inline uint32_t sum_blocks(const hq::Fp8Sums &s) { return s.parts ? static_cast<uint32_t>((s.columns + 15) / 16) : 0; }

}  // namespace
