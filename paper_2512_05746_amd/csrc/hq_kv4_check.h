// The host's checks of a cache and a call's tokens, shared by the calls on 4-bit caches.
#pragma once
#include "hq_common.h"
#include "hq_fp8.h"
#include "hq_kv4.h"

namespace hq {

inline bool is_pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

inline hq_status kv4_check(const hq_kv4 &a, int heads, Kv4 *out) {
    if (a.kv_heads <= 0 || a.d <= 0 || a.d % 8 || a.batch < 0 || a.table_pages <= 0 || a.pages <= 0 || a.t < 0 || heads <= 0) return HQ_ERR_SHAPE;
    if (heads % a.kv_heads || !is_pow2(a.page_size) || !is_pow2(a.had_block) || a.d % a.had_block) return HQ_ERR_SHAPE;
    if (a.batch == 0 ? a.t != 0 : !a.begins && a.t % a.batch) return HQ_ERR_SHAPE;
    if (a.d > 256 || a.page_size < 8 || a.had_block > 128) return HQ_ERR_UNSUPPORTED;
    if (a.table_pages > 0x7FFF0000 / a.page_size || a.t > 0x7FFF0000 / (heads + 1) || a.batch > 0x03FFFFFF || a.t > 0x3FFFFFFF)
        return HQ_ERR_UNSUPPORTED;
    if (a.t / 8 + 2 * int64_t{a.batch} > 0x500000) return HQ_ERR_UNSUPPORTED;   // groups: three workgroups each are one launch
    // (a page's place is its number times what a page takes of codes, both of 32 bits)
    if (a.pages > 0x7FFFFFFF || int64_t{a.page_size} * a.kv_heads > 0xFFFFFFFFll / 128) return HQ_ERR_UNSUPPORTED;
    if (a.t > 0 && (!a.k || !a.v || !a.k_scale || !a.v_scale || !a.page_table || !a.lengths)) return HQ_ERR_NULL;
    if (!aligned16(a.k) || !aligned16(a.v) || !aligned16(a.k_scale) || !aligned16(a.v_scale)) return HQ_ERR_ALIGN;
    if (!aligned_to(a.page_table, 4) || !aligned_to(a.lengths, 4) || !aligned_to(a.begins, 4)) return HQ_ERR_ALIGN;
    *out = Kv4{a.k, a.v, a.k_scale, a.v_scale, a.page_table, a.lengths, a.begins, a.pages, ilog2(a.page_size), a.kv_heads, a.d, kv4_pitch(a.d),
               ilog2(a.had_block), a.batch, a.table_pages, static_cast<int>(a.t), a.batch ? static_cast<int>(a.t / a.batch) : 0};
    return HQ_OK;
}

}  // namespace hq
