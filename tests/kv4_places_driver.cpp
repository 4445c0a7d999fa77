// Where the calls on a 4-bit cache look and what they work on, for arrays that say sensible things and for arrays that do not.  CPU only.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "hq_kv4.h"

using namespace hq;

static long bad = 0;
#define EXPECT(x, ...)                            \
    do {                                          \
        if (!(x) && ++bad <= 10) {                \
            std::printf("%s: ", #x);              \
            std::printf(__VA_ARGS__);             \
            std::printf("\n");                    \
        }                                         \
    } while (0)

struct Call {
    std::vector<int32_t> table, lengths, begins;
    Kv4 c{};
};

static int sequence_of(const Kv4 &c, int index) {   // as a wave counts it
    int s = -1;
    for (int b = 0; b <= c.batch; ++b) s += kv4_group_begin(c.begin(b), b) <= index;
    return std::max(s, 0);
}

static void finish(Kv4Cut &cut) {
    cut.reach = kv4_reach(cut.window, cut.sinks, cut.rows(), cut.group);
    // as the host's exact division of numbers below 2^31: m = ceil(2^(31 + l) / d), l = ceil(log2 d)
    uint32_t l = 0;
    while ((1ull << l) < static_cast<uint64_t>(cut.group)) ++l;
    cut.magic = cut.group > 1 ? static_cast<uint32_t>(((1ull << (31 + l)) + cut.group - 1) / cut.group) : 0;
    cut.shift = l ? l - 1 : 0;
    for (const int row : {0, 1, cut.group - 1, cut.group, 1000003, 0x7FFEFFFF, 0x7FFFFFFF})
        EXPECT(cut.token_of(row) == row / cut.group, "row %d of groups of %d", row, cut.group);
}

// every group lies inside the call; a token is in one group where begins rises
static void groups(const Call &call, bool sound) {
    const Kv4 &c = call.c;
    std::vector<int> seen(c.t);
    for (int i = 0; i < kv4_groups(c.t, c.batch); ++i) {
        const int s = sequence_of(c, i);
        EXPECT(s <= c.batch, "%d", s);
        if (!c.begins) EXPECT(kv4_sequence(c, i) == s, "group %d: sequence %d, not %d", i, kv4_sequence(c, i), s);
        const Kv4Group g = kv4_group(c, s, c.begin(s), c.begin(std::min(s + 1, c.batch)), i, [](const int32_t *p) { return *p; });
        EXPECT(g.count >= 0 && g.count <= 8 && g.row >= 0 && g.row + g.count <= c.t, "row %d, count %d of %d", g.row, g.count, c.t);
        if (g.count <= 0 || g.row < 0 || g.row + g.count > c.t) continue;
        for (int r = 0; r < g.count; ++r) ++seen[g.row + r];
        if (g.s >= c.batch) continue;
        EXPECT((g.position >> 3) == ((g.position + g.count - 1) >> 3), "position %d, count %d", g.position, g.count);
        const int n = c.begin(s + 1) - c.begin(s);
        EXPECT(int64_t{g.position} == int64_t{std::max(0, c.lengths[s])} - n + (g.row - c.begin(s)), "position %d", g.position);
        const int64_t page = c.page(s, g.position);
        EXPECT(page >= -1 && page < c.pages, "page %lld", static_cast<long long>(page));
        EXPECT(page < 0 || (g.position >= 0 && g.position + g.count <= c.capacity()), "position %d of %d", g.position, c.capacity());
        if (page >= 0) EXPECT(c.slot(g.position) + g.count <= 1 << c.page_log2, "a group crosses a page");
    }
    if (sound)
        for (int t = 0; t < c.t; ++t) EXPECT(seen[t] == 1, "token %d is in %d groups", t, seen[t]);
}

// tasks stay below what the host allots; every row's visible tokens are in its tiles
static void tasks(const Call &call, const Kv4Cut &cut, bool sound) {
    const Kv4 &c = call.c;
    float work = 0.0f;
    for (int s = 0; s < c.batch; ++s) {
        const Kv4Span p = kv4_span(c, cut, s);
        EXPECT(p.begin >= 0 && p.n >= 0 && p.begin + int64_t{p.n} <= c.t && p.steps >= 0 && p.steps <= c.capacity() / 32 + 1, "span");
        work += static_cast<float>(p.blocks) * static_cast<float>(p.steps);
    }
    const int part = kv4_part(cut, work, c.kv_heads);
    EXPECT(part >= cut.least, "part %d", part);
    int64_t blocks = 0, slots = 0;
    for (int s = 0; s < c.batch; ++s) {
        const Kv4Span p = kv4_span(c, cut, s);
        const int parts = kv4_parts(p, part);
        EXPECT(parts >= 1, "parts %d", parts);
        blocks += int64_t{p.blocks} * parts * c.kv_heads;
        if (parts > 1) slots += int64_t{p.blocks} * parts * c.kv_heads;
        if (p.length > c.capacity()) continue;   // (answered with NaN)
        const int rows = p.n * cut.group;
        for (int b = 0; b < p.blocks; ++b)
            for (const int per : {cut.rows(), cut.rows() >> cut.waves_log2}) {   // a workgroup's rows, and a wave's
                for (int row0 = b * cut.rows(); row0 < std::min((b + 1) * cut.rows(), rows); row0 += per) {
                    const int last_row = std::min(row0 + per, rows) - 1, base = p.length - p.n;
                    const Kv4Tiles t = kv4_tiles(base + row0 / cut.group, base + last_row / cut.group, cut.window, cut.sinks);
                    EXPECT(t.sinks >= 0 && t.sinks <= t.from + (t.count() == 0) && t.from <= t.to && t.to * int64_t{32} < int64_t{p.length} + 32, "tiles %d %d %d of %d", t.sinks, t.from, t.to, p.length);
                    std::vector<char> in(p.length / 32 + 2);
                    for (int i = 0; i < t.count(); ++i) {
                        EXPECT(t.tile(i) * 32 < p.length, "tile %d", t.tile(i));
                        EXPECT(!in[t.tile(i)], "tile %d twice", t.tile(i));
                        in[t.tile(i)] = 1;
                    }
                    for (int row = row0; row <= last_row; row += std::max(1, cut.group)) {
                        const int pos = base + row / cut.group;
                        for (int j = 0; j <= pos; ++j) {
                            const bool visible = cut.window == 0 || j > pos - int64_t{cut.window} || j < cut.sinks;
                            const Kv4Seen seen = kv4_seen(pos, cut.window, cut.sinks);
                            EXPECT(visible == (j >= seen.from || j < seen.sinks), "place %d for %d", j, pos);
                            if (visible) EXPECT(in[j / 32], "place %d for %d, window %d, sinks %d", j, pos, cut.window, cut.sinks);
                        }
                    }
                }
            }
    }
    if (sound) {
        const int64_t most = int64_t{c.kv_heads} * (int64_t{c.t} * cut.group / cut.rows() + c.batch);
        EXPECT(blocks <= most + cut.target, "%lld workgroups, %lld allotted", static_cast<long long>(blocks), static_cast<long long>(most + cut.target));
        EXPECT(slots <= 2 * int64_t{cut.target}, "%lld slots of %d", static_cast<long long>(slots), 2 * cut.target);
    }
}

int main() {
    std::mt19937 rng(7);
    const auto below = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
    long calls = 0;
    for (int turn = 0; turn < 4000; ++turn, ++calls) {
        Call call;
        Kv4 &c = call.c;
        const bool sound = turn % 4 != 0;
        c.page_log2 = 3 + below(4);
        c.batch = 1 + below(turn % 5 ? 6 : 70);
        c.table_pages = 1 + below(12);
        c.pages = 1 + below(40);
        c.kv_heads = 1 + below(4);
        c.d = 64, c.pitch = 64;
        const bool uniform = below(3) == 0;
        const int capacity = c.table_pages << c.page_log2;
        for (int b = 0; b < c.batch; ++b) call.lengths.push_back(sound ? below(capacity + 1) : below(2) ? static_cast<int32_t>(rng()) : below(3 * capacity) - capacity);
        call.begins.push_back(sound || below(2) ? 0 : static_cast<int32_t>(rng()));
        c.each = uniform ? below(40) : 0;
        for (int b = 0; b < c.batch; ++b)
            call.begins.push_back(sound ? call.begins.back() + (below(3) ? below(30) : 0) : below(2) ? static_cast<int32_t>(rng()) : below(200) - 20);
        c.t = uniform ? c.each * c.batch : sound ? call.begins.back() + below(20) : below(200);
        for (int i = 0; i < c.batch * c.table_pages; ++i)
            call.table.push_back(sound ? below(static_cast<int>(c.pages)) : below(2) ? static_cast<int32_t>(rng()) : below(60) - 10);
        c.table = call.table.data(), c.lengths = call.lengths.data(), c.begins = uniform ? nullptr : call.begins.data();
        groups(call, sound || uniform);
        Kv4Cut cut{};
        cut.waves_log2 = 2 + below(2), cut.rows_log2 = 4 + cut.waves_log2 + below(2), cut.group = 1 + below(9), cut.target = 1 + below(64), cut.least = 1 + below(8);
        cut.window = below(2) ? 1 + below(100) : 0, cut.sinks = cut.window ? below(70) : 0;
        finish(cut);
        tasks(call, cut, sound || uniform);
    }
    // the ends of the range: lengths near 2^31, a table that does not reach
    for (const int32_t length : {0x7FFFFFFF, 0x7FFF0000, -0x7FFFFFFF - 1}) {
        Call call;
        Kv4 &c = call.c;
        call.table = {0}, call.lengths = {length}, call.begins = {0, 16};
        c.table = call.table.data(), c.lengths = call.lengths.data(), c.begins = call.begins.data();
        c.page_log2 = 4, c.batch = 1, c.table_pages = 1, c.pages = 1, c.kv_heads = 1, c.d = 64, c.pitch = 64, c.t = 16;
        groups(call, true);
        Kv4Cut cut{6, 2, 4, 8, 1, 0, 0, 0, 0, 0};
        finish(cut);
        tasks(call, cut, true);
    }
    // places beyond 32 bits of bytes
    Kv4 c{};
    c.page_log2 = 6, c.kv_heads = 8, c.d = c.pitch = 128, c.pages = int64_t{1} << 24;
    EXPECT((c.slots(c.pages - 1, 7) + 63) * c.row_bytes() == ((((int64_t{1} << 24) * 8) << 6) - 1) * 64, "slots");
    std::printf("%ld calls, %ld bad\n", calls, bad);
    return bad != 0;
}
