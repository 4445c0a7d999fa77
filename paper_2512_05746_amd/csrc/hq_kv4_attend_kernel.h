// Attention over a 4-bit cache.  For a key head of one sequence, the rows are its new tokens times the query heads that share it:
//
//     s_rj = scale q_r k_j = scale (H q_r) . (codes of k_j) x k_scale_j,   o_r = H sum_j p_rj v_scale_j (codes of v_j) / sum_j p_rj
//
// with p the exponential of s minus a reference that follows the largest s so far: one pass over the cache.
//
// A wave holds tiles of 16 rows and takes 32 tokens a turn, all in registers: 4-bit codes turn into halves by one instruction for two,
// exactly, so that they go from memory to the matrix instruction without LDS.  Products are taken the other way round,
// S^T = K Q^T and O^T = V^T P^T: then a lane has one row of the tile throughout (its reference, its sum, its factor need no exchange), and the
// weights that leave the first product are in the lanes and in the order in which the second one takes them, if row m of the first tile of
// 16 tokens is token 8 (m / 4) + m % 4 and of the second 4 further on.  v is kept channel by channel for 8 tokens, the order of its operand.
//
// Roundings: H q to half (2^-11 of an element), in units of a power of two that leaves the row's largest below 2^12; weights times v_scale to
// half, the largest v_scale so far times the weight of the reference as 2^6 to 2^7 (2^-11; below 2^-20 of it, 2^-31 of it).  For half and 32-bit
// results H q is two halves (2^-22; a rounding of q moves every score of its row, and results were off by twice their own rounding), for
// 32-bit ones the weights too.  Codes are exact, sums are 32 bits.
//
// The reference moves only where s would exceed it by 8 (by 2 for 32-bit results), so most turns leave the sums alone.
//
// What bounds it (medians of a kernel trace).  A few rows over many tokens: the cache's bytes (276 MB for 64 sequences of up to 16384 tokens, 32 query
// and 8 key heads of 128: 67 us, 4.1 TB/s; a copy reaches 5.1 to 5.4).  Prompts: a turn's instructions (825 GF for 2 sequences of 4096 new tokens over
// 8192, the same heads: 930 to 1000 us from card to card, 820 to 890 TF/s, 867 at best; a large library product in bf16 reaches 1540): 32 products of 7.7 ns
// beside about 200 vector instructions, which overlap with those of the SIMD's other wave in part only (the vector pipe is busy two thirds of the time,
// the matrix pipe a third).  One row over few tokens: latencies, 13.6 us: about 1 until a workgroup knows its work, 4 to 5 until its rows are through
// the transform (with the first k and v under way), 2 a turn, of which pages below 32 tokens wait for all of k (below), 2 to 3 for the results.
// Taken back for prompts: the next tile's products beside this one's exponentials (1016 -> 1068 us), k and v asked for two tiles ahead (1110 to
// 1130), scales one a lane and moved to where they are used (slower by the moves), three waves a SIMD (spills).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hq_floats.h"
#include "hq_kv4_attend.h"
#include "hq_kv4_lanes.h"

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

// Sums over the lanes before and with one, by moves inside rows of 16 lanes and from a row's last lane on.
template <class T, int CTRL, int ROWS>
__device__ __forceinline__ T moved(T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
template <class T>
__device__ __forceinline__ T wave_prefix(T v) {
    v += moved<T, 0x111, 0xF>(v);
    v += moved<T, 0x112, 0xF>(v);
    v += moved<T, 0x114, 0xF>(v);
    v += moved<T, 0x118, 0xF>(v);
    v += moved<T, 0x142, 0xA>(v);
    v += moved<T, 0x143, 0xC>(v);
    return v;
}
// (of numbers that are not negative)
__device__ __forceinline__ int wave_max(int v) {
    v = max(v, moved<int, 0x111, 0xF>(v));
    v = max(v, moved<int, 0x112, 0xF>(v));
    v = max(v, moved<int, 0x114, 0xF>(v));
    v = max(v, moved<int, 0x118, 0xF>(v));
    v = max(v, moved<int, 0x142, 0xA>(v));
    v = max(v, moved<int, 0x143, 0xC>(v));
    return __builtin_amdgcn_readlane(v, 63);
}
template <class T>
__device__ __forceinline__ T lane_value(T v, int lane) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
template <class T>
__device__ __forceinline__ T wave_sum(T v) { return lane_value(wave_prefix(v), 63); }
// What the wave's lanes wrote to LDS, to be read by each other.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// The sequences' spans, a lane each; the first 64 are kept.
struct Spans {
    const hq::Kv4Attend &a;
    const int lane;
    const hq::Kv4Span first;
    __device__ __forceinline__ Spans(const hq::Kv4Attend &a, int lane) : a(a), lane(lane), first(read(0)) {}
    __device__ __forceinline__ hq::Kv4Span read(int from) const {
        return from + lane < a.c.batch ? hq::kv4_span(a.c, a.cut, from + lane) : hq::Kv4Span{};
    }
    __device__ __forceinline__ hq::Kv4Span at(int from) const { return from ? read(from) : first; }
    // Steps of a part: every wave adds up the work by itself, in the same order.
    __device__ __forceinline__ int part() const {
        if (!a.split) return hq::kKv4Undivided;
        float work = 0.0f;
        for (int from = 0; from < a.c.batch; from += 64) {
            const hq::Kv4Span p = at(from);
            work += wave_sum(static_cast<float>(p.blocks) * static_cast<float>(p.steps));
        }
        return hq::kv4_part(a.cut, work, a.c.kv_heads);
    }
};
__device__ __forceinline__ hq::Kv4Span of_lane(const hq::Kv4Span &p, int lane) {
    return {lane_value(p.begin, lane), lane_value(p.n, lane), lane_value(p.length, lane), lane_value(p.blocks, lane), lane_value(p.steps, lane)};
}

// What a workgroup works on: a part of the tokens of a block of rows of one key head.  The last blocks of a sequence, which see most, come
// first, and of 64 sequences the long ones: what begins late is to end soon (12 sequences of 10 to 700 tokens, 576 workgroups of which 512 are
// at work at once: 63 -> 57 us).  The heads of a block follow one another, so that eight heads go to the eight XCDs and each finds its own in its
// cache.
struct Task {
    int s, head, block, part, parts, slot;   // slot: its place among the parts' sums; s = -1: none, and `block` counts up from 0
    hq::Kv4Span span;
};
__device__ __forceinline__ Task task_of(const hq::Kv4Attend &a, int id, int lane) {
    const Spans spans(a, lane);
    const int part = spans.part();
    int base = 0, slots = 0;
    for (int from = 0; from < a.c.batch; from += 64) {
        const hq::Kv4Span p = spans.at(from);
        const int parts = a.split ? hq::kv4_parts(p, part) : 1;
        const int count = p.blocks * parts * a.c.kv_heads, mine = parts > 1 ? count : 0;
        const int steps = count ? hq::kv4_min(p.steps, part) : 0, longest = wave_max(steps);
        const int count_long = 2 * int64_t{steps} > longest ? count : 0, to_long = wave_prefix(count_long);
        const int all_long = lane_value(to_long, 63), slot_to = a.split ? wave_prefix(mine) : 0;
        const bool is_long = base + all_long > id;
        const int to = is_long ? to_long : all_long + wave_prefix(count - count_long);
        const uint64_t behind = __ballot(base + to > id);
        if (behind) {
            const int at = __ffsll(static_cast<unsigned long long>(behind)) - 1;
            Task t;
            t.span = of_lane(p, at);
            const unsigned in = id - base - lane_value(to - (is_long ? count_long : count - count_long), at), of = lane_value(parts, at);
            const unsigned row_blocks = of == 1 ? in : in / of;
            t.s = from + at;
            t.slot = slots + lane_value(slot_to - mine, at) + in;
            t.parts = of;
            t.part = in - row_blocks * of;
            const unsigned turn = row_blocks / static_cast<unsigned>(a.c.kv_heads);
            t.head = row_blocks - turn * a.c.kv_heads;
            t.block = t.span.blocks - 1 - turn;
            return t;
        }
        base += lane_value(to, 63);
        slots += lane_value(slot_to, 63);
    }
    Task none{};
    none.s = -1;
    none.block = id - base;
    return none;
}

template <class F>
__device__ __forceinline__ void with_type(hq_dtype dt, F f) {
    if (dt == HQ_F16) f(static_cast<_Float16 *>(nullptr));
    else if (dt == HQ_BF16) f(static_cast<__bf16 *>(nullptr));
    else f(static_cast<float *>(nullptr));
}

// A row's result: its sums back through the transform, 8 channels a lane.
template <int KS>
__device__ __forceinline__ void store_row(const hq::Kv4Attend &a, float (&o)[8], float weight, int in, int64_t at) {
    const bool live = in * 8 < a.c.d;
    const float f = weight == 0.0f ? 0.0f : walsh_factor(in, a.c.block_log2) / weight;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = live && weight != 0.0f ? o[i] : 0.0f;
    walsh(o, in, a.c.block_log2);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= f;
    if (live) with_type(a.dtype, [&](auto *t) { store8(static_cast<decltype(t)>(a.out) + at + in * 8, o); });
}
template <int KS>
__device__ __forceinline__ void store_all(const hq::Kv4Attend &a, float value, int in, int64_t at) {
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = value;
    if (in * 8 < a.c.d) with_type(a.dtype, [&](auto *t) { store8(static_cast<decltype(t)>(a.out) + at + in * 8, o); });
}

constexpr int lanes_of(int ks) { return ks <= 1 ? 4 : ks <= 2 ? 8 : ks <= 4 ? 16 : 32; }   // that own a row, 8 channels each

// 32 tokens as they are in memory.
template <int KS> struct Turn {
    uint32_t k[2][KS], v[2 * KS];
    float4v ks[2], vs[2];
    bool bad;   // the lane's group of tokens has no page
};
template <int N>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t *w) {
    typedef uint32_t words __attribute__((ext_vector_type(N == 3 ? 3 : N >= 4 ? 4 : N), aligned(4)));
    constexpr int STEP = N >= 4 ? 4 : N;
    const words t = *reinterpret_cast<const words *>(p);
#pragma unroll
    for (int i = 0; i < STEP; ++i) {
        if constexpr (N == 1) w[i] = __builtin_bit_cast(uint32_t, t);
        else w[i] = t[i];
    }
    if constexpr (N > STEP) load_words<N - STEP>(p + 4 * STEP, w + STEP);
}
// The largest of 8 numbers that are not NaN, by instructions that take three (written out: fmaxf comes with an instruction more for each
// operand, in case it is a signalling NaN).
__device__ __forceinline__ float largest(const float (&v)[8]) {
    float x, y;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(x) : "v"(v[0]), "v"(v[1]), "v"(v[2]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(y) : "v"(v[3]), "v"(v[4]), "v"(v[5]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(x) : "v"(x), "v"(v[6]), "v"(v[7]));
    asm("v_max_f32 %0, %1, %2" : "=v"(x) : "v"(x), "v"(y));
    return x;
}
// Waves a SIMD for which registers are kept: loads of other waves and conversions beside products need them.  (One tile of rows: bound by loads,
// more waves, for which heads of 128 channels keep 9 to 11 registers in scratch memory outside the loop over tokens; two tiles: their sums and queries
// alone are 96 registers at 96 channels.)
constexpr int waves_of(int ks, int r, int qh, int waves) { return waves == 8 ? 2 : r == 1 && ks <= 4 ? qh == 1 ? 4 : 3 : ks <= 6 ? 2 : 1; }
// Of a tile's groups of 8 tokens the lane's: one for all, or one of four.
template <class T, int N>
__device__ __forceinline__ T of_group(const T (&x)[N], int part) {
    if constexpr (N == 1) return x[0];
    else return part & 2 ? (part & 1 ? x[3] : x[2]) : (part & 1 ? x[1] : x[0]);
}
// Row m of the products with v has, of each 64 channels, 4 (2 in a last part of 32): lanes that follow one another read what follows one another.
// Lane m's channel number e.
template <int KS>
__device__ __forceinline__ constexpr int channel_of(int m, int e) {
    return e / 4 * 64 + (2 * KS - e / 4 * 4 < 4 ? 2 : 4) * m + e % 4;
}
template <int N>
__device__ __forceinline__ void load_channels(const uint8_t *p, int m, uint32_t *w) {
    constexpr int STEP = N < 4 ? N : 4;
    load_words<STEP>(p + m * (4 * STEP), w);
    if constexpr (N > STEP) load_channels<N - STEP>(p + 256, m, w + STEP);
}
// Conversions and products in the order in which they are written: four conversions, then the products that take them.  (Left to itself the
// compiler converts everything first, in registers that the sums need.)
template <int N, int PRODUCTS>
__device__ __forceinline__ void order() {
    if constexpr (N > 0) {
        __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, PRODUCTS, 0);
        order<N - 1, PRODUCTS>();
    }
}
// By how much a score may exceed the reference, as a power of two: less where weights are two halves, whose second ones want the room.
constexpr int lazy_of(int ph) { return ph > 1 ? 2 : 8; }
// Weights times v_scale are kept 2^room as large as the reference says, next to the end of a half (2^room 2 2^lazy = 2^15): below 2^-14 a half
// has fewer bits, and over long sequences most weights are small (32-bit results over 3001 tokens: 2.6e-6 off without room, 3.5 to 6e-7 with 2^6).
constexpr int room_of(int ph) { return 14 - lazy_of(ph); }
template <bool B> using Flag = std::integral_constant<bool, B>;

// R tiles of 16 rows a wave, WAVES waves a workgroup; a tile of k and v is converted once for R products.  Rows that fill more than one wave's
// tiles: rows of its own for each wave.  Otherwise all waves have the same rows, and tiles of 32 tokens in turn.  QH, PH: halves for an element of
// H q, for a weight.  WIDE_PAGES: pages of 32 tokens or more, so that a tile's place is one number for the wave.
template <int KS, int R, int WAVES, int QH, int PH, bool WIDE_PAGES>
__global__ __launch_bounds__(64 * WAVES, waves_of(KS, R, QH, WAVES)) void attend_kernel(hq::Kv4Attend a) {
    constexpr int DP = 32 * KS, LP = lanes_of(KS), STAGE = DP + 8, ROW = DP + 4;
    // per wave: a tile of rows as halves, and later their sums
    constexpr int WAVE_BYTES = 16 * ROW * 4 > 16 * STAGE * 2 * QH ? 16 * ROW * 4 : 16 * STAGE * 2 * QH;
    __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES][WAVE_BYTES];
    __shared__ float row_factor[R][WAVES][16], row_top[WAVES][16], row_sum[WAVES][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const Task task = task_of(a, blockIdx.x, lane);
    const int in = kv4_block(lane % LP);   // the 8 channels that the lane has where a row is dealt to lanes
    if (task.s < 0) {
        // rows of no sequence: zeros
        if (task.block < 0) return;   // (begins that do not rise can ask for more work than can be counted)
        const int begin = a.c.begin(a.c.batch), rows = (a.c.t - begin) * a.heads;
        const int64_t from = int64_t{blockIdx.x} - task.block, step = (int64_t{gridDim.x} - from) * (64 * WAVES / LP);
        for (int64_t r = int64_t{task.block} * (64 * WAVES / LP) + threadIdx.x / LP; r < rows; r += step) {
            const int row = static_cast<int>(r);
            store_all<KS>(a, 0.0f, in, (begin + row / a.heads) * a.out_token + row % a.heads * a.out_head);
        }
        return;
    }
    const int s = task.s, head = task.head;
    const hq::Kv4Span &span = task.span;
    if (head >= a.c.kv_heads || (task.parts > 1 && task.slot >= a.slots)) return;
    const int group = a.cut.group, rows = span.n * group;   // (below 2^31: the host checks t x heads)
    const bool apart = rows - (task.block << a.cut.rows_log2) <= 16 * R;   // tokens are apart, not rows (in a sequence's last block too)
    const int row0 = (task.block << a.cut.rows_log2) + (apart ? 0 : wave * 16 * R);
    const int by = apart ? 64 * WAVES / LP : 64 / LP, mine_at = apart ? threadIdx.x / LP : lane / LP;   // rows at once, this lane's
    const auto at_of = [&](int row, int64_t by_token, int64_t by_head) {
        const int token = a.cut.token_of(row);
        return (span.begin + token) * by_token + (head * group + row - token * group) * by_head;
    };
    if (span.length > a.c.capacity()) {   // the sequence says that it has tokens that no page holds
        if (task.part == 0)
            for (int r = mine_at; r < 16 * R && row0 + r < rows; r += by)
                store_all<KS>(a, __builtin_nanf(""), in, at_of(row0 + r, a.out_token, a.out_head));
        return;
    }
    // ---- the tokens: the first of them are asked for before the rows are prepared
    const int last_row = hq::kv4_min(row0 + 16 * R, rows) - 1;
    const int first_position = span.length - span.n + a.cut.token_of(row0),
              last_position = row0 < rows ? span.length - span.n + a.cut.token_of(last_row) : -1;
    const hq::Kv4Tiles tiles = hq::kv4_tiles(first_position, last_position, a.cut.window, a.cut.sinks);
    const int seen_from = hq::kv4_seen(last_position, a.cut.window, a.cut.sinks).from;
    const int step = apart ? WAVES : 1;
    int share = tiles.count();
    if (task.parts > 1) share = (share + task.parts * step - 1) / (task.parts * step) * step;
    const int end = hq::kv4_min(tiles.count(), (task.part + 1) * share);
    int i = task.part * share + (apart ? wave : 0);

    // Where the tokens of a tile are, by scalar loads of the table: vector loads arrive in order, so that waiting for one of these would
    // mean waiting for every k and v that was asked for before it.  Groups of 8 tokens have one place each, tiles of wide pages one.  (Scalar
    // instructions take the wave's turns too: a place is two multiplications of 32 bits, from what one head's page begins with.)
    // With narrow pages a lane's choice of four places becomes an indexed load from scratch memory (80 bytes a lane; LDS in the kernels of 8 waves from 160
    // channels on), which arrives in that order as well: there the next k has arrived before v is asked for.
    constexpr int GROUPS = WIDE_PAGES ? 1 : 4;
    const uint32_t page_slots = static_cast<uint32_t>(a.c.kv_heads) << a.c.page_log2, page_bytes = page_slots * (DP / 2);
    const uint32_t pages = static_cast<uint32_t>(a.c.pages);
    const int64_t head_slot = static_cast<int64_t>(head) << a.c.page_log2;
    const uint8_t *const k_head = a.c.k + head_slot * (DP / 2), *const v_head = a.c.v + head_slot * (DP / 2);
    const uint8_t *const ks_head = reinterpret_cast<const uint8_t *>(a.c.k_scale + head_slot);
    const uint8_t *const vs_head = reinterpret_cast<const uint8_t *>(a.c.v_scale + head_slot);
    struct Place {
        uint64_t codes[GROUPS], scales[GROUPS];   // in bytes
        bool none[GROUPS];                        // without a page: the first page is read, and dropped
    };
    const auto *const table = reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(
        reinterpret_cast<uint64_t>(a.c.table + static_cast<int64_t>(s) * a.c.table_pages));
    // An entry is asked for a turn before it is looked at.
    struct Entries {
        uint32_t of[GROUPS];
    };
    const auto entries_of = [&](int index) {
        const int first = tiles.tile(index) * 32;
        Entries p;
#pragma unroll
        for (int e = 0; e < GROUPS; ++e) {
            const int column = (first + 8 * e) >> a.c.page_log2;
            p.of[e] = table[WIDE_PAGES ? column : hq::kv4_min(column, a.c.table_pages - 1)];   // (a wide tile begins inside the sequence)
        }
        return p;
    };
    const auto place_of = [&](int index, const Entries &entries) {
        const int first = tiles.tile(index) * 32;
        Place p;
#pragma unroll
        for (int e = 0; e < GROUPS; ++e) {
            const uint32_t slot = a.c.slot(first + 8 * e);
            p.none[e] = entries.of[e] >= pages || (!WIDE_PAGES && first + 8 * e >= a.c.capacity());   // (a negative one is large)
            const uint32_t page = p.none[e] ? 0 : entries.of[e];
            p.codes[e] = static_cast<uint64_t>(page) * page_bytes + slot * (DP / 2);
            p.scales[e] = static_cast<uint64_t>(page) * (page_slots * 4) + slot * 4;
        }
        return p;
    };
    Turn<KS> turn;
    const uint32_t k_lane = ((WIDE_PAGES ? 8 * (m >> 2) : 0) + (m & 3)) * (DP / 2) + g * (KS * 4);
    const uint32_t v_lane = WIDE_PAGES ? g * (DP * 4) : 0, scale_lane = WIDE_PAGES ? g * 32 : 0;
    const auto load_k = [&](const Place &p) {
        const uint8_t *const k = k_head + of_group(p.codes, m >> 2) + k_lane;
        const uint8_t *const ks = ks_head + of_group(p.scales, g) + scale_lane;
        turn.bad = of_group(p.none, g);
        load_words<KS>(k, turn.k[0]);
        load_words<KS>(k + 4 * (DP / 2), turn.k[1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) turn.ks[e] = reinterpret_cast<const float4v *>(ks)[e];
    };
    const auto load_v = [&](const Place &p) {
        const uint8_t *const vs = vs_head + of_group(p.scales, g) + scale_lane;
        load_channels<2 * KS>(v_head + of_group(p.codes, g) + v_lane, m, turn.v);
#pragma unroll
        for (int e = 0; e < 2; ++e) turn.vs[e] = reinterpret_cast<const float4v *>(vs)[e];
    };
    // ---- the rows are asked for, then the first k and v (by waves without tokens too: loads under way are counted in order, and what the
    // compiler cannot count it waits for), so that the rows are prepared while these are on their way
    using T = std::conditional_t<(PH > 1), float, std::conditional_t<(QH > 1), _Float16, __bf16>>;
    constexpr int PASSES = LP / 4;   // of a wave through a tile's rows; of all waves fewer
    typename Vec<T, 8>::type raw[R][PASSES];
    const int begin = i < end ? i : 0;
    Entries entries = entries_of(begin);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            const int i2 = mine_at + pass * by, row = row0 + 16 * r + i2;
            raw[r][pass] = typename Vec<T, 8>::type{};
            if (i2 < 16 && row < rows && in * 8 < a.c.d)
                raw[r][pass] = load_vec<T, 8>(static_cast<const T *>(a.q) + at_of(row, a.q_token, a.q_head) + in * 8);
        }
    __builtin_amdgcn_sched_barrier(0);
    // k of a turn is asked for when the products with k of the turn before are done, v likewise; its place a turn before that
    {
        const Place place = place_of(begin, entries);
        load_k(place);
        load_v(place);
        entries = entries_of(begin + step < end ? begin + step : begin);
    }
    __builtin_amdgcn_sched_barrier(0);
    // through the transform, to halves, to the lanes of the matrix instruction
    half8v q[R][QH][KS];
    float factor[R];
    int position[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (apart && r) __syncthreads();
        const int owner = apart ? 0 : wave;
        uint8_t *const stage = lds[owner];
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            const int i2 = mine_at + pass * by;
            if (i2 >= 16) break;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(raw[r][pass][e]);
            walsh(x, in, a.c.block_log2);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
            top = max_lanes<LP>(top);
            // x = x' 2^power, |x'| < 2^12: halves of full precision down to 2^-26 of the largest; smaller for a row so small that its factor would
            // be below 2^-126 (masked scores are -infinity, and that times 0 is NaN)
            int power = top == 0 || top >= 0x7F800000u ? 0 : __builtin_amdgcn_frexp_expf(__uint_as_float(top)) - 12;
            power = max(power, -125 - __builtin_amdgcn_frexp_expf(a.scale));
            float f = __builtin_ldexpf(a.scale, power);
            const float sign = a.scale == 0.0f ? 0.0f : (walsh_factor(in, a.c.block_log2) < 0.0f) != (a.negative != 0) ? -1.0f : 1.0f;
            if (a.scale == 0.0f) f = 1.0f;
            if (top >= 0x7F800000u) f = __builtin_nanf("");
            half8v hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = top >= 0x7F800000u ? 0.0f : __builtin_ldexpf(x[e], -power) * sign;
                hi[e] = static_cast<_Float16>(y);
                lo[e] = static_cast<_Float16>(y - static_cast<float>(hi[e]));
            }
            if (in * 8 < DP) {
                *reinterpret_cast<half8v *>(stage + (i2 * STAGE + in * 8) * 2) = hi;
                if constexpr (QH > 1) *reinterpret_cast<half8v *>(stage + (16 * STAGE + i2 * STAGE + in * 8) * 2) = lo;
            }
            if (in == 0) row_factor[r][owner][i2] = f;
        }
        if (apart) __syncthreads();
        else wave_sync();
#pragma unroll
        for (int h = 0; h < QH; ++h)
#pragma unroll
            for (int e = 0; e < KS; ++e) q[r][h][e] = *reinterpret_cast<const half8v *>(stage + (h * 16 * STAGE + m * STAGE + g * (DP / 4) + e * 8) * 2);
        factor[r] = row_factor[r][owner][m];
        const int row = row0 + 16 * r + m;
        position[r] = row < rows ? span.length - span.n + a.cut.token_of(row) : -1;
        if (!apart) wave_sync();
    }

    constexpr int LAZY = lazy_of(PH), ROOM = room_of(PH);
    float4v o[R][2 * KS];
    float top[R], sum[R];                  // the reference, this lane's sum of weights
    float most_allowed[R], minus[R];       // what moves the reference, its negative (0 for none)
    // The largest v_scale that the reference allows for, and its power of two less ROOM: up to 48 of that are in the reference, so that weights and their
    // sums stay normal numbers down to 2^-78 of the largest and parts can be joined, the rest is taken from v_scale and is in o only.
    float limit = 0.0f, power = -48.0f;
    int v_power = -1000, rest = 0;
    // Scores beyond 2^16 are rounded before the reference is taken from them (in the multiply-add that takes it from the exact product the largest
    // would be left with what its own rounding was, as a power of two), the reference is the largest, and all of v's power is in rest.
    int far = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        top[r] = most_allowed[r] = -__builtin_inff();
        minus[r] = sum[r] = 0.0f;
#pragma unroll
        for (int e = 0; e < 2 * KS; ++e) o[r][e] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (; i < end; i += step) {
        const int first = tiles.tile(i) * 32, next = i + step < end ? i + step : i;   // (the last turn asks for its own tile again)
        float4v t[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) t[r][0] = t[r][1] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < KS; ++e)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const half8v k = kv4_halves(turn.k[h][e]);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int l = QH - 1; l >= 0; --l) t[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[r][l][e], t[r][h], 0, 0, 0);
            }
        order<2 * KS, R * QH>();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            t[r][0] *= turn.ks[0];
            t[r][1] *= turn.ks[1];
        }
        const bool bad = turn.bad;
        __builtin_amdgcn_sched_barrier(0);
        const Place place = place_of(next, entries);
        load_k(place);
        __builtin_amdgcn_sched_barrier(0);
        float scale_v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) scale_v[e] = turn.vs[e >> 2][e & 3];
        const bool whole = first + 31 <= first_position && (first >= seen_from || first + 32 <= a.cut.sinks) && !__any(bad);
        if (!whole || far) {
            const int token = first + 8 * g;
            if (far) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float f = row_factor[r][apart ? 0 : wave][m];
                    t[r][0] *= f;
                    t[r][1] *= f;
                }
            }
            // A scale of v that is not finite makes the scores of the rows that see its token NaN instead, so that it does not meet the weight 0
            // of those that do not; behind the sequence's end scales are whatever the page held.
            uint32_t odd = bad ? 0xFFu : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float &x = scale_v[e];
                if (!(fabsf(x) < __builtin_inff())) odd |= 1u << e;
                if (odd >> e & 1 || token + e >= span.length) x = 0.0f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int from = a.cut.window > 0 && position[r] >= a.cut.window ? position[r] - a.cut.window + 1 : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = token + e;
                    const bool seen = j <= position[r] && (j >= from || j < a.cut.sinks);
                    t[r][e >> 2][e & 3] = seen ? odd >> e & 1 ? __builtin_nanf("") : t[r][e >> 2][e & 3] : -__builtin_inff();
                }
            }
        }
        float most[R];
        const float v_most = largest(scale_v);
        bool move = v_most >= limit;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float all[8] = {t[r][0][0], t[r][0][1], t[r][0][2], t[r][0][3], t[r][1][0], t[r][1][1], t[r][1][2], t[r][1][3]};
            most[r] = largest(all) * factor[r];
            move |= most[r] > most_allowed[r];
        }
        if (__ballot(move) | static_cast<uint32_t>(rest)) {
            float v_top = fmaxf(v_most, __shfl_xor(v_most, 16));
            v_top = fmaxf(v_top, __shfl_xor(v_top, 32));
            if (v_top >= limit && v_top > 0.0f) {
                v_power = hq::kv4_max(v_power, __builtin_amdgcn_frexp_expf(v_top) - 1 - ROOM);
                limit = __builtin_ldexpf(2.0f, v_power + ROOM);   // (infinite for the largest)
            }
            float to[R];
            bool large = false;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float here = fmaxf(most[r], __shfl_xor(most[r], 16));
                here = fmaxf(here, __shfl_xor(here, 32));
                to[r] = fmaxf(top[r] - power, here);
                large |= fabsf(to[r]) > 0x1p16f && fabsf(to[r]) < __builtin_inff();
            }
            if (!far && __any(large)) {
                far = 1;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    t[r][0] *= factor[r];
                    t[r][1] *= factor[r];
                    factor[r] = 1.0f;
                }
            }
            const int in_reference = far ? 0 : hq::kv4_max(-48, hq::kv4_min(48, v_power)), before = rest;
            power = static_cast<float>(in_reference);
            rest = __builtin_amdgcn_readfirstlane(v_power == -1000 ? 0 : v_power - in_reference);   // (v's scales are the same for all rows)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float ahead = to[r] + power;
                const float f = top[r] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top[r] - ahead);
                top[r] = ahead;
                most_allowed[r] = far ? to[r] : to[r] + LAZY;
                minus[r] = ahead == -__builtin_inff() ? 0.0f : -ahead;
                sum[r] *= f;
                const float of_o = __builtin_ldexpf(f, before - rest);
#pragma unroll
                for (int e = 0; e < 2 * KS; ++e) o[r][e] *= of_o;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) scale_v[e] = __builtin_ldexpf(scale_v[e], -rest);
        }
        half8v p[R][PH];
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(t[r][e >> 2][e & 3], factor[r], minus[r]));
                float y = w * scale_v[e];
                // (the compiler would round the exact product to the first half, by an instruction that does both, and y for the second: next to
                // a tie they would not belong together)
                if constexpr (PH > 1) asm("" : "+v"(y));
                sum[r] += w;
                p[r][0][e] = static_cast<_Float16>(y);
                if constexpr (PH > 1) p[r][1][e] = static_cast<_Float16>(y - static_cast<float>(p[r][0][e]));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 2 * KS; ++e) {
            const half8v v = kv4_halves(turn.v[e]);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int l = PH - 1; l >= 0; --l) o[r][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[r][l], o[r][e], 0, 0, 0);
        }
        order<2 * KS, R * PH>();
        __builtin_amdgcn_sched_barrier(0);
        load_v(place);
        __builtin_amdgcn_sched_barrier(0);
        entries = entries_of(i + 2 * step < end ? i + 2 * step : next);
    }
    if (rest) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 2 * KS; ++e)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[r][e][c] = __builtin_ldexpf(o[r][e][c], rest);
    }
    // ---- the waves' sums together, and out
#pragma unroll
    for (int r = 0; r < R; ++r) {
        sum[r] += __shfl_xor(sum[r], 16);
        sum[r] += __shfl_xor(sum[r], 32);
        if (apart) __syncthreads();
        else wave_sync();
        float *const mine = reinterpret_cast<float *>(lds[wave]);
        // lane (m, g) has, of row m, the channels of rows 4 g + e of the products
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < 2 * KS; c += 2) {
                *reinterpret_cast<float2v *>(mine + m * ROW + channel_of<KS>(4 * g + e, c)) = float2v{o[r][c][e], o[r][c + 1][e]};
            }
        if (g == 0) {
            row_top[wave][m] = top[r];
            row_sum[wave][m] = sum[r];
        }
        if (apart) __syncthreads();
        else wave_sync();
        for (int i2 = mine_at; i2 < 16; i2 += by) {
            const int row = row0 + 16 * r + i2;
            if (row >= rows) continue;
            float x[8], weight, reference;
            if (apart) {
                reference = row_top[0][i2];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) reference = fmaxf(reference, row_top[w][i2]);
                weight = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = row_top[w][i2] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(row_top[w][i2] - reference);
                    weight += f * row_sum[w][i2];
                    if (in * 8 < DP) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] += f * reinterpret_cast<const float *>(lds[w])[i2 * ROW + in * 8 + e];
                    }
                }
            } else {
                reference = row_top[wave][i2];
                weight = row_sum[wave][i2];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = in * 8 < DP ? mine[i2 * ROW + in * 8 + e] : 0.0f;
            }
            if (span.length - span.n + a.cut.token_of(row) < 0) weight = 0.0f;   // (it sees nothing, whatever its query is)
            if (task.parts == 1) {
                store_row<KS>(a, x, weight, in, at_of(row, a.out_token, a.out_head));
            } else {
                const int64_t at = (int64_t{task.slot} << a.cut.rows_log2) + (apart ? 0 : wave * 16 * R) + 16 * r + i2;
                if (in * 8 < DP) store8(a.sums + at * DP + in * 8, x);
                if (in == 0) {
                    a.tops[2 * at] = reference;
                    a.tops[2 * at + 1] = weight;
                }
            }
        }
    }
}

// The parts of rows' tokens together: a workgroup for a token and as many heads as it has slots of lanes (EACH), or for one of them, whose
// parts the slots share.
template <int KS, bool EACH>
__global__ __launch_bounds__(256) void join_kernel(hq::Kv4Attend a) {
    constexpr int DP = 32 * KS, LP = lanes_of(KS), SLOTS = 256 / LP;
    const int lane = threadIdx.x & 63, token = blockIdx.x, in = kv4_block(threadIdx.x % LP), slot = threadIdx.x / LP;
    const int q_head = EACH ? blockIdx.y * SLOTS + slot : blockIdx.y;
    const Spans spans(a, lane);
    const int part = spans.part();
    int s = -1, slots = 0;
    for (int from = 0; from <= a.c.batch; from += 64) {
        const int at = from + lane;
        const bool before = at <= a.c.batch && a.c.begin(at) <= token;
        s += __popcll(__ballot(before));
    }
    if (s >= a.c.batch) return;
    s = __builtin_amdgcn_readfirstlane(s);
    // (of sequences without tokens the last one that begins here)
    const hq::Kv4Span span = s < 64 ? of_lane(spans.first, s) : hq::kv4_span(a.c, a.cut, s);
    const int parts = hq::kv4_parts(span, part);
    if (parts == 1 || span.length > a.c.capacity()) return;
    for (int from = 0; from < s; from += 64) {
        const hq::Kv4Span p = spans.at(from);
        const int of = hq::kv4_parts(p, part);
        slots += wave_sum(from + lane < s && of > 1 ? p.blocks * of * a.c.kv_heads : 0);
    }
    if (q_head >= a.heads) return;   // (EACH: no lane waits for another slot's)
    const int group = a.cut.group, head = a.cut.token_of(q_head), row = (token - span.begin) * group + q_head - head * group;
    const int64_t before = int64_t{slots} + ((span.blocks - 1 - (row >> a.cut.rows_log2)) * int64_t{a.c.kv_heads} + head) * parts;
    if (before < 0 || before + parts > a.slots) return;
    const int64_t first = (before << a.cut.rows_log2) + (row & (a.cut.rows() - 1));
    float x[8], top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    const auto add = [&](float other_top, float other_sum, const float (&other)[8]) {
        if (other_sum == 0.0f) return;   // (a row that is NaN has no reference, but a sum)
        const float to = fmaxf(top, other_top);
        const float mine = top == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top - to), by = __builtin_amdgcn_exp2f(other_top - to);
        top = to;
        sum = sum * mine + other_sum * by;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * mine + other[e] * by;
    };
    // four parts at a time: their loads are under way together
    constexpr int STEP = EACH ? 1 : SLOTS;
    for (int p = EACH ? 0 : slot; p < parts; p += 4 * STEP) {
        float y[4][8], tops[4], sums[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int there = p + i * STEP < parts ? p + i * STEP : p;
            const int64_t at = first + (int64_t{there} << a.cut.rows_log2);
            tops[i] = a.tops[2 * at];
            sums[i] = there == p && i ? 0.0f : a.tops[2 * at + 1];
            load8(a.sums + at * DP + (in * 8 < DP ? in * 8 : 0), y[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) add(tops[i], sums[i], y[i]);
    }
    if constexpr (!EACH) {
        __shared__ float x_of[SLOTS][LP * 8 + 4], top_of[SLOTS], sum_of[SLOTS];
#pragma unroll
        for (int e = 0; e < 8; ++e) x_of[slot][in * 8 + e] = x[e];
        if (in == 0) {
            top_of[slot] = top;
            sum_of[slot] = sum;
        }
        __syncthreads();
        if (slot) return;
        for (int p = 1; p < SLOTS && p < parts; ++p) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x_of[p][in * 8 + e];
            add(top_of[p], sum_of[p], y);
        }
    }
    store_row<KS>(a, x, sum, in, token * a.out_token + q_head * a.out_head);
}

}  // namespace

namespace hq {

template <int KS>
void kv4_attend_launch(const Kv4Attend &a, Kv4Shape shape, unsigned blocks, hipStream_t st) {
    const auto go = [&](auto tiles, auto waves, auto q_halves, auto p_halves, auto wide_pages) {
        constexpr int R = decltype(tiles)::value, WAVES = decltype(waves)::value;
        attend_kernel<KS, R, WAVES, decltype(q_halves)::value, decltype(p_halves)::value, decltype(wide_pages)::value><<<blocks, 64 * WAVES, 0, st>>>(a);
    };
    const auto with_pages = [&](auto tiles, auto waves, auto q_halves, auto p_halves) {
        if (a.c.page_log2 >= 5) go(tiles, waves, q_halves, p_halves, Flag<true>{});
        else go(tiles, waves, q_halves, p_halves, Flag<false>{});
    };
    const auto with_halves = [&](auto tiles, auto waves) {
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        if (a.dtype == HQ_F32) with_pages(tiles, waves, two, two);
        else if (a.dtype == HQ_F16) with_pages(tiles, waves, two, one);
        else with_pages(tiles, waves, one, one);
    };
    if (shape.waves == 8) with_halves(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
    else if (shape.tiles == 1) with_halves(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
    else if constexpr (KS <= 4) with_halves(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
    if (!a.split) return;
    // (many rows have few parts: 2177 tokens of 16 heads, 2 to 4 parts: a workgroup for a row 45 us, for 8 or 16 rows 7; few rows have many parts:
    // a row's parts are read side by side, 64 tokens of 32 heads 6.5 us)
    constexpr int SLOTS = 256 / lanes_of(KS);
    if (int64_t{a.c.t} * a.heads > 8192) join_kernel<KS, true><<<dim3(a.c.t, (a.heads + SLOTS - 1) / SLOTS), 256, 0, st>>>(a);
    else join_kernel<KS, false><<<dim3(a.c.t, a.heads), 256, 0, st>>>(a);
}

}  // namespace hq
