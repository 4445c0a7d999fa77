// Every lane of every cut of a head: what it reads of a token's row of the tables, and which channels it has.  CPU only.
#include <cstdio>
#include <vector>

#include "hq_qk_cut.h"

int main() {
    long bad = 0, lanes = 0;
    for (int d = 2; d <= 1024; d += 2)
        for (int rotary = 0; rotary <= d; rotary += 2)
            for (const hq_dtype dt : {HQ_F16, HQ_F32})
                for (const bool back : {false, true})
                    for (const bool interleaved : {false, true}) {
                        const hq::QkCut cut = hq::qk_cut_of(d, rotary, dt, back);
                        if (!cut.g) continue;   // (a wave for a head: pairs one by one, each compared with their count)
                        std::vector<int> owners(d);
                        for (int in = 0; in < cut.g; ++in, ++lanes) {
                            const hq::QkLane l = hq::qk_lane_of(d, rotary, interleaved, cut.c, in);
                            bool ok = l.at.first >= 0 && l.at.first + cut.c <= d && l.at.second >= 0 && l.at.second + cut.c <= d;
                            if (l.at.rotated) ok = ok && l.p >= 0 && l.p + cut.c <= rotary / 2;
                            if (!ok && ++bad <= 10)
                                std::printf("d %d, rotary %d, type %d, back %d, interleaved %d, lane %d of %d: table %d .. %d of %d\n", d, rotary, dt, back,
                                            interleaved, in, cut.g, l.p, l.p + cut.c - 1, rotary / 2);
                            for (int i = 0; ok && l.live && i < cut.c; ++i) ++owners[l.at.first + i], ++owners[l.at.second + i];
                        }
                        for (int c = 0; c < d; ++c)
                            if (owners[c] != 1 && ++bad <= 10) std::printf("d %d, rotary %d: channel %d has %d owners\n", d, rotary, c, owners[c]);
                    }
    std::printf("%ld lanes, %ld bad\n", lanes, bad);
    return bad != 0;
}
