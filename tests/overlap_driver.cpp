// Shared memory of two strided views, against marking every byte.  CPU only.
#include <cstdio>
#include <random>
#include <vector>

#include "hq_overlap.h"

static bool marked(const hq::Rows2 &a, const hq::Rows2 &b) {
    std::vector<char> byte(4096);
    for (int64_t i = 0; i < a.n[0]; ++i)
        for (int64_t j = 0; j < a.n[1]; ++j)
            for (int64_t c = 0; c < a.bytes; ++c) byte[a.at + i * a.stride[0] + j * a.stride[1] + c] = 1;
    for (int64_t i = 0; i < b.n[0]; ++i)
        for (int64_t j = 0; j < b.n[1]; ++j)
            for (int64_t c = 0; c < b.bytes; ++c)
                if (byte[b.at + i * b.stride[0] + j * b.stride[1] + c]) return true;
    return false;
}

int main() {
    std::mt19937 gen(1);
    const auto pick = [&](int low, int high) { return static_cast<int64_t>(low + gen() % (high - low + 1)); };
    int bad = 0, shared = 0, apart = 0, inside = 0;
    for (int k = 0; k < 400000; ++k) {
        hq::Rows2 v[2];
        for (hq::Rows2 &r : v) r = {pick(0, 120), {pick(0, 6), pick(0, 5)}, {pick(0, 60), pick(0, 60)}, pick(1, 12)};
        if (k % 2) v[1].stride[0] = v[0].stride[0];   // as views of one buffer have them
        if (k % 4 == 3) v[1].stride[1] = v[0].stride[1];
        const bool want = marked(v[0], v[1]);
        if (want) ++shared;
        else if (v[0].empty() || v[1].empty() || v[0].end() <= v[1].at || v[1].end() <= v[0].at) ++apart;
        else ++inside;
        for (int swap = 0; swap < 2; ++swap)
            if (hq::rows_overlap(v[swap], v[1 - swap]) != want && ++bad <= 5) {
                for (const hq::Rows2 &r : v)
                    std::printf("at %d: %d x %d rows of %d, %d and %d apart\n", int(r.at), int(r.n[0]), int(r.n[1]), int(r.bytes), int(r.stride[0]),
                                int(r.stride[1]));
                std::printf("shared: %d\n", want);
            }
    }
    std::printf("%d shared, %d apart, %d between each other; %d wrong\n", shared, apart, inside, bad);
    return bad != 0 || shared < 1000 || apart < 1000 || inside < 1000;
}
