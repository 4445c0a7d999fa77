// Attention over a 4-bit cache: what the kernels (hq_kv4_attend_kernel.h) and the entry point (hq_kv4_attend.hip) share.
#pragma once
#include <hip/hip_runtime.h>

#include "hq_kv4.h"

namespace hq {

struct Kv4Attend {
    Kv4 c;
    Kv4Cut cut;
    const void *q;
    void *out;
    int64_t q_token, q_head, out_token, out_head;   // strides, in elements
    hq_dtype dtype;
    int heads;
    float scale;     // of q k, in powers of two: its magnitude, with the transform's factor
    int negative;    // scale is negative
    int split;       // parts of a row's tokens may be apart: their sums go to `sums`
    int slots;       // (a call whose begins do not rise could ask for more: those parts are left out)
    float *sums;     // [slots, rows, pitch]
    float *tops;     // [slots, rows, 2]: the reference that a part's sums are relative to, the sum of its weights
};

// Tiles of 16 rows a wave, waves a workgroup.
struct Kv4Shape {
    int tiles, waves;
    int rows() const { return 16 * tiles * waves; }
};
// One launch for heads of up to 32 KS channels (hq_kv4_attend_<..>.hip).
template <int KS> void kv4_attend_launch(const Kv4Attend &a, Kv4Shape shape, unsigned blocks, hipStream_t st);

}  // namespace hq
