// A model of the dense layer kernels' pipeline on the CPU: two producers in one or two CTAs, an MMA warp that frees stages,
// copies that land when they like, and barriers with arrival and byte counts.  At a random moment every role stops, as it
// does when a bounded wait is given up; then the barriers are supplied with what is missing (csrc/unwind.cuh), the
// remaining copies land in a random order, and whoever waits for the barriers must find them complete exactly when
// nothing is on its way any more.  Prints the number of trials in which that fails; with "naive" the wait covers the
// uses of the leader's A alone, which the model has to show to be too few.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../paper_2506_11728_b200/csrc/unwind.cuh"

struct Barrier {
    int count = 0, pending = 0, phase = 0;
    long tx = 0;
    void init(int n) { count = pending = n; }
    void settle() {
        if (pending == 0 && tx == 0) { ++phase; pending = count; }
    }
    void arrive(long expect) { tx += expect; --pending; settle(); }
    void complete(long bytes) { tx -= bytes; settle(); }
};
struct Copy { uint32_t use; int cta, operand; long bytes; };

int main(int argc, char** argv) {
    const bool naive = argc > 1 && !std::strcmp(argv[1], "naive");
    std::mt19937 rng(argc > 2 ? std::atoi(argv[2]) : 1);
    const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
    int failures = 0, uneven = 0;
    const int trials = 20000;
    for (int trial = 0; trial < trials; ++trial) {
        const int ctas = 1 + pick(2), operands = 1 + pick(2);
        const uint32_t stages = 2 + pick(5), total = 1 + pick(30);
        const uint32_t bytes[2] = {1000u + pick(5000), 1000u + pick(5000)};
        std::vector<Barrier> full(stages);
        for (auto& b : full) b.init(operands);
        uint32_t issued[2][2] = {{0, 0}, {0, 0}}, consumed = 0;
        std::vector<Copy> flying;
        const auto land = [&] {
            if (flying.empty()) return;
            const int i = pick(static_cast<int>(flying.size()));
            const Copy c = flying[i];
            flying.erase(flying.begin() + i);
            full[c.use % stages].complete(c.bytes);
        };
        for (int step = pick(300); step > 0; --step) {
            const int what = pick(8);
            if (what < 4) {                              // a producer asks for its next use, if its stage is free
                const int cta = what / 2 % ctas, o = what % operands;
                uint32_t& n = issued[cta][o];
                if (n >= total || n >= consumed + stages) continue;
                if (cta == 0) full[n % stages].arrive(static_cast<long>(bytes[o]) * ctas);
                flying.push_back(Copy{n, cta, o, bytes[o]});
                ++n;
            } else if (what < 6) {
                land();
            } else if (consumed < total && full[consumed % stages].phase > static_cast<int>(consumed / stages)) {
                ++consumed;                              // the MMA warp has read a stage
            }
        }
        // everybody has stopped
        uint32_t last = 0;
        for (int c = 0; c < ctas; ++c)
            for (int o = 0; o < operands; ++o) {
                last = mip::uses_last(last, issued[c][o]);
                if (issued[c][o] != issued[0][0]) ++uneven;
            }
        if (naive) last = issued[0][0];
        const uint32_t first = mip::uses_first(last, stages);
        if (!naive)
            for (uint32_t use = first; use < last; ++use)
                for (int o = 0; o < operands; ++o) {
                    const mip::MissingCopy m = mip::missing_copy(use, issued[0][o], issued[ctas - 1][o], bytes[o]);
                    if (m.complete) full[use % stages].complete(m.complete);
                    if (m.arrive) full[use % stages].arrive(m.expect);
                }
        const auto complete = [&](uint32_t use) { return full[use % stages].phase > static_cast<int>(use / stages); };
        bool ok = true;
        while (true) {
            bool all = true;
            for (uint32_t use = first; use < last; ++use) all = all && complete(use);
            if (all) {
                ok = ok && flying.empty();               // the wait is over: nothing may be on its way
                break;
            }
            if (flying.empty()) { ok = false; break; }   // nothing will come any more: the wait would run out
            land();
        }
        // no barrier may have been driven past the use that was waited for
        for (uint32_t s = 0; ok && !naive && s < stages; ++s) {
            int want = 0;
            for (uint32_t use = s; use < last; use += stages) ++want;
            ok = full[s].phase == want;
        }
        failures += !ok;
    }
    std::printf("%d %d %d\n", failures, uneven, trials);
    return 0;
}
