// Attention over a 4-bit cache: the entry point, and how its work is cut.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "hq_common.h"
#include "hq_fp8.h"
#include "hq_kv4_attend.h"
#include "hq_kv4_check.h"

namespace {

struct Plan {
    hq::Kv4Shape shape;
    hq::Kv4Cut cut;
    bool split;
    int64_t blocks, slots;
};
// How rows and tokens are dealt to workgroups:
//   Sequences of up to 16 rows on average, and heads of more than 128 channels (whose second tile of rows would spill): one tile of rows a wave.
//     Otherwise two: a tile of k and v is converted once for both (12 sequences of 10 to 700 tokens, 16 heads of 80: one 76 us, two 62).
//   8 waves share the tokens of a row where that leaves no CU without work and the table has room for at most 2048 of them (lengths are
//     known on the device only, so the table's width stands for them, here and below; it was measured on tables as wide as their
//     sequences): 13.8 us for 777 tokens of 8 key heads, 4 waves 15.8, 16 waves 17.
//   Tokens are divided where rows alone do not fill the card and are more than 12 turns of the waves (below, the second launch costs more than
//     it saves), into as many parts as are at work at once, at least 8 turns each.  For two tiles half as many again were slower
//     (57 -> 68 us), twice as many too.
Plan plan_of(const hq::Kv4 &c, int heads, hq_dtype dtype, int window, int sinks) {
    const int group = heads / c.kv_heads, cus = hq::compute_units();
    const int64_t rows = c.batch ? (int64_t{c.t} * group + c.batch - 1) / c.batch : 0;   // of a sequence, on average
    Plan p;
    const bool few = rows <= 16 || c.pitch > 128;
    const int64_t items = int64_t{c.kv_heads} * std::max<int64_t>(1, c.batch);
    p.shape = few ? hq::Kv4Shape{1, items <= cus && rows <= 16 && c.capacity() <= 2048 ? 8 : 4} : hq::Kv4Shape{2, 4};
    const int64_t most = int64_t{c.kv_heads} * (int64_t{c.t} * group / p.shape.rows() + c.batch);   // blocks of rows
    const int target = (p.shape.tiles == 1 ? 3 : 2) * cus;   // workgroups of 4 waves that a CU holds
    const int64_t tokens = window > 0 ? std::min<int64_t>(c.capacity(), int64_t{window} + sinks + 64) : c.capacity();
    const hq::Magic31 m = hq::magic31(group);
    p.cut = hq::Kv4Cut{hq::ilog2(p.shape.rows()), hq::ilog2(p.shape.waves), group, target, 8, window, sinks,
                       hq::kv4_reach(window, sinks, p.shape.rows(), group), m.m, m.s};
    p.split = tokens > 12 * 32 * (p.shape.tiles == 1 && rows <= 16 ? p.shape.waves : 1) && most < target;
    p.blocks = most + (p.split ? target : 0) + 1;
    p.slots = p.split ? 2 * (target + int64_t{c.kv_heads}) : 0;
    return p;
}
int64_t bytes_of(const Plan &p, int d) { return p.slots * p.shape.rows() * (hq::kv4_pitch(d) + 2) * 4; }

}  // namespace

extern "C" int64_t hq_kv4_attention_workspace(const hq_kv4 *cache, hq_dtype dtype, int heads, int window, int sinks) {
    hq::Kv4 c;
    if (!cache || !hq::is_float(dtype) || hq::kv4_check(*cache, heads, &c) != HQ_OK || window < 0 || sinks < 0) return 0;
    return bytes_of(plan_of(c, heads, dtype, window, sinks), c.d);
}

extern "C" hq_status hq_kv4_attention(const hq_kv4 *cache, const void *q, hq_dtype dtype, int heads, const int64_t *strides, float scale,
                                      int window, int sinks, void *workspace, void *out, void *stream) {
    if (!cache || !strides) return HQ_ERR_NULL;
    if (!hq::is_float(dtype)) return HQ_ERR_DTYPE;
    hq::Kv4 c;
    if (const hq_status s = hq::kv4_check(*cache, heads, &c)) return s;
    if (c.t > 0 && (!q || !out)) return HQ_ERR_NULL;
    if (window < 0 || sinks < 0 || !(fabsf(scale) <= 0x1p100f)) return HQ_ERR_SHAPE;
    if (!hq::aligned_to(q, hq::size_of(dtype)) || !hq::aligned_to(out, hq::size_of(dtype))) return HQ_ERR_ALIGN;
    if (c.t == 0) return HQ_OK;
    if (window == 0) sinks = 0;
    const Plan p = plan_of(c, heads, dtype, window, sinks);
    if (p.blocks * 64 * p.shape.waves > 0xFFFFFFFFll) return HQ_ERR_UNSUPPORTED;   // lanes of a launch
    if (p.slots && !workspace) return HQ_ERR_NULL;
    if (!hq::aligned16(workspace)) return HQ_ERR_ALIGN;
    hq::Kv4Attend a{};
    a.c = c;
    a.cut = p.cut;
    a.q = q;
    a.out = out;
    a.q_token = strides[0], a.q_head = strides[1], a.out_token = strides[2], a.out_head = strides[3];
    a.dtype = dtype;
    a.heads = heads;
    a.scale = static_cast<float>(fabs(static_cast<double>(scale)) * 1.4426950408889634 * pow(2.0, -0.5 * c.block_log2));
    a.negative = scale < 0.0f;
    a.split = p.split;
    a.slots = static_cast<int>(p.slots);
    a.sums = static_cast<float *>(workspace);
    a.tops = a.sums + p.slots * p.shape.rows() * c.pitch;
    const hq::LaunchCheck check;
    const auto st = static_cast<hipStream_t>(stream);
    const auto blocks = static_cast<unsigned>(p.blocks);
    switch (c.pitch / 32) {
        case 1: hq::kv4_attend_launch<1>(a, p.shape, blocks, st); break;
        case 2: hq::kv4_attend_launch<2>(a, p.shape, blocks, st); break;
        case 3: hq::kv4_attend_launch<3>(a, p.shape, blocks, st); break;
        case 4: hq::kv4_attend_launch<4>(a, p.shape, blocks, st); break;
        case 5: hq::kv4_attend_launch<5>(a, p.shape, blocks, st); break;
        case 6: hq::kv4_attend_launch<6>(a, p.shape, blocks, st); break;
        case 7: hq::kv4_attend_launch<7>(a, p.shape, blocks, st); break;
        default: hq::kv4_attend_launch<8>(a, p.shape, blocks, st); break;
    }
    return check.status();
}
