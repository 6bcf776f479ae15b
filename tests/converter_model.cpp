// A model of the product kernel's codes, converters and products on the CPU: barriers with phases, of which a waiter tests
// the parity alone; a producer that asks for the codes of use after use; copies that land in any order; two groups of
// converter warps that take the uses in turn, each waiting in the order of csrc/stage_waits.h; an MMA warp.  Prints the
// number of uses converted from codes of another use, with the waits in the kernel's order or ("swapped") in the other.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../paper_2506_11728_b200/csrc/stage_waits.h"

struct Barrier {
    int count, pending, phase = 0;
    explicit Barrier(int n) : count(n), pending(n) {}
    void arrive() { if (--pending == 0) { ++phase; pending = count; } }
    bool done(int parity) const { return (phase & 1) != parity; }       // the phase of that parity is the last one completed
};

int main(int argc, char** argv) {
    const bool swapped = argc > 1 && !std::strcmp(argv[1], "swapped");
    std::mt19937 rng(argc > 2 ? std::atoi(argv[2]) : 1);
    const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
    const mip::StageWait order[2] = {swapped ? mip::kConverterSecond : mip::kConverterFirst, swapped ? mip::kConverterFirst : mip::kConverterSecond};
    long wrong = 0, uses = 0, stuck = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        const int stages = 2 + pick(5), total = 40;
        std::vector<Barrier> codes(stages, Barrier(1)), codes_read(stages, Barrier(1)), converted(stages, Barrier(1)), free_(stages, Barrier(1));
        std::vector<int> holds(stages, -1), flying;
        int asked = 0, products = 0;
        struct Group { int it, step; } group[2] = {{0, 0}, {1, 0}};
        int idle = 0;
        while (products < total && idle < 100000) {
            ++idle;
            const int what = pick(5);
            if (what == 0 && asked < total) {                            // producer: the codes' buffer has been read
                const int st = asked % stages, ph = asked / stages & 1;
                if (!codes_read[st].done(ph ^ 1)) continue;
                flying.push_back(asked++);
            } else if (what == 1 && !flying.empty()) {                   // a copy lands
                const int i = pick(static_cast<int>(flying.size())), use = flying[i];
                flying.erase(flying.begin() + i);
                holds[use % stages] = use;
                codes[use % stages].arrive();
            } else if (what == 2 || what == 3) {                         // a group goes on: wait, wait, convert
                Group& g = group[what - 2];
                if (g.it >= total) continue;
                const int st = g.it % stages, ph = g.it / stages & 1;
                if (g.step < 2) {
                    if (order[g.step] == mip::kStageFree ? free_[st].done(ph ^ 1) : codes[st].done(ph)) ++g.step;
                    continue;
                }
                wrong += holds[st] != g.it;
                ++uses;
                converted[st].arrive();
                codes_read[st].arrive();
                g.it += 2;
                g.step = 0;
            } else if (what == 4) {                                      // products of the next use, then its stage is free
                const int st = products % stages;
                if (!converted[st].done(products / stages & 1)) continue;
                free_[st].arrive();
                ++products;
            }
        }
        stuck += products < total;
    }
    std::printf("%ld %ld %ld\n", wrong, stuck, uses);
    return 0;
}
