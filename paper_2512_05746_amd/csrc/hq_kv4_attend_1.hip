// Attention over a 4-bit cache: heads of up to 32 channels.
#include "hq_kv4_attend_kernel.h"
template void hq::kv4_attend_launch<1>(const hq::Kv4Attend &, hq::Kv4Shape, unsigned, hipStream_t);
