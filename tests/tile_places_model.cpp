// A model, on the CPU, of how far apart the warps of the dense 8-bit floating-point product may be: barriers with phases, of which a
// waiter tests the parity alone; the scales' warp, which may go on while the products of `depth` blocks before are ready; the
// tensor core's warp, whose products of a block are done some time later; two summing warps for each half of the tile, which read a
// block's scales, give its buffer back and, behind a tile's last block, look up where the tile lies.  Every role goes at a speed of its
// own, drawn for each trial.
//   model DEPTH HALVES BLOCKS RING SEED [PLACES BEHIND]
// BLOCKS of K in a tile; RING: entries that the scales' warp hands tile positions over in; PLACES: for the scales of that many blocks
// (2 * DEPTH); BEHIND: 1, the last of a block's scales are read behind the buffer's return, else in front of it.  Prints the tiles whose
// position had been written over when it was read, the trials that did not end, the tiles, and the blocks whose scales had been written
// over when they were read.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

struct Barrier {
    int count, pending, phase = 0;
    explicit Barrier(int n) : count(n), pending(n) {}
    void arrive() { if (--pending == 0) { ++phase; pending = count; } }
    bool done(int parity) const { return (phase & 1) != parity; }       // the phase of that parity is the last one completed
};

int main(int argc, char** argv) {
    if (argc < 6) return 2;
    const int depth = std::atoi(argv[1]), halves = std::atoi(argv[2]), blocks = std::atoi(argv[3]), ring = std::atoi(argv[4]);
    std::mt19937 rng(std::atoi(argv[5]));
    const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
    const int places = argc > 6 ? std::atoi(argv[6]) : 2 * depth;
    const bool behind = argc > 7 && std::atoi(argv[7]) != 0;
    constexpr int kTiles = 24, kWarps = 2;
    long moved = 0, stuck = 0, tiles = 0, wrong = 0;
    for (int trial = 0; trial < 2000; ++trial) {
        const int total = kTiles * blocks, roles = 3 + kWarps * halves;
        std::vector<std::vector<Barrier>> ready(halves, std::vector<Barrier>(depth, Barrier(2)));
        std::vector<std::vector<Barrier>> given(halves, std::vector<Barrier>(depth, Barrier(kWarps)));
        std::vector<int> where(ring, -1), scales(places, -1), speed(roles);
        for (int& s : speed) s = 1 << pick(6);
        // scales: block and half it waits for; products: issued, and of those done; summing warps: block, step
        int scale_block = 0, scale_half = 0, issued = 0, finished = 0;
        bool scale_told = false;
        struct Warp { int block = 0, step = 0; };
        std::vector<Warp> warps(kWarps * halves);
        const auto over = [&] { for (const Warp& w : warps) if (w.block < total) return false; return true; };
        long idle = 0;
        while (!over() && idle < 4000000) {
            ++idle;
            const int role = pick(roles);
            if (pick(32) >= speed[role]) continue;
            if (role == 0) {                                             // the scales' warp
                if (scale_block >= total) continue;
                if (scale_block % blocks == 0 && !scale_told) {          // (a tile's position, before any wait for the tile)
                    where[scale_block / blocks % ring] = scale_block / blocks;
                    scale_told = true;
                    continue;
                }
                const int acc = scale_block % depth, use = scale_block / depth;
                if (use > 0 && !ready[scale_half][acc].done((use - 1) & 1)) continue;
                if (++scale_half < halves) continue;
                scales[scale_block % places] = scale_block;
                for (int h = 0; h < halves; ++h) ready[h][acc].arrive();
                scale_half = 0;
                ++scale_block;
                scale_told = false;
            } else if (role == 1) {                                      // products of a half of a block are asked for
                if (issued >= total * halves) continue;
                const int b = issued / halves, h = issued % halves, acc = b % depth, use = b / depth;
                if (given[h][acc].done((use & 1) ^ 1)) ++issued;
            } else if (role == 2) {                                      // ... and done, in their order
                if (finished < issued) {
                    ready[finished % halves][finished / halves % depth].arrive();
                    ++finished;
                }
            } else {
                Warp& w = warps[role - 3];
                if (w.block >= total) continue;
                const int h = (role - 3) / kWarps, acc = w.block % depth, use = w.block / depth;
                if (w.step == 0) {                                       // products and scales are there
                    if (!ready[h][acc].done(use & 1)) continue;
                    w.step = 1;
                    wrong += scales[w.block % places] != w.block;
                } else if (w.step == 1) {                                // read: the buffer is given back
                    if (!behind) wrong += scales[w.block % places] != w.block;
                    given[h][acc].arrive();
                    w.step = 2;
                } else {                                                 // behind the last block, the tile's outputs
                    if (behind) wrong += scales[w.block % places] != w.block;
                    if ((w.block + 1) % blocks == 0) {
                        const int t = w.block / blocks;
                        moved += where[t % ring] != t;
                        ++tiles;
                    }
                    ++w.block;
                    w.step = 0;
                }
            }
        }
        stuck += !over();
    }
    std::printf("%ld %ld %ld %ld\n", moved, stuck, tiles, wrong);
    return 0;
}
