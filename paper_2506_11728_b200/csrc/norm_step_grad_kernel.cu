// The step between two blocks of a transformer layer, backward: from the gradients of y and h those of x, z, the gate and
// the norms' weights and biases.  With ^ for a normalised value and q, p for the reciprocal deviations of the two norms:
//     g = dy + q (w dh - mean(w dh) - y^ mean(w dh y^)),   dx = s g,
//     k = mask g,   dgate = sum k u,   m = gate k,   dz = p (w' m - mean(w' m) - z^ mean(w' m z^))
// (the first means for a norm that subtracts its mean only), and over all rows dw = sum dh y^, db = sum dh,
// dw' = sum m z^, db' = sum m.  The rows' statistics come from the forward pass, so each norm needs one exchange; the mask
// is drawn again from its counter.
//
// Workers (CTAs, or clusters of CTAs that share a row of more than 8192 columns) go through the rows, 16 columns a thread; a second
// kernel adds the workers' column sums in a fixed order.  Rows are dealt in units that lie within one gate row, so that a
// unit's sum is a share of one row of dgate.  The column sums lie in shared memory, where each thread has places of its own:
// in registers (40 to 80 of a thread's) they left room for one block on an SM, whose warps waited for each row's exchanges
// together; two blocks by turns, with the next row's elements on their way, fill those gaps.
//
// What bounds it: the instructions (1000 of a warp for 16 columns of a row with two norms, a gate and dropout) and their latencies,
// beside the bytes of dy, dh, y, z, dx and dz: 16384 x 4096 bf16 238 to 241 us, the bytes 123.  Gate rows that few rows share leave most
// of a CTA's rows side by side idle (16384 x 1024, a gate for 2 rows 143 us, for each row 69); rows that take a whole cluster wait for
// its barriers (4096 x 16384 337 us, 4096 x 32768 1111, the bytes 246).
#include <algorithm>
#include <atomic>

#include "ptx.cuh"
#include "step_math.cuh"

namespace mip {

namespace {

constexpr int kGradThreads = 512, kBlockThreads = 256;       // most threads of a row's CTA; of a CTA with several rows side by side
constexpr int kGradRuns = 2, kGradCols = 8 * kGradRuns;      // columns per thread
constexpr int kMaxGradRows = kBlockThreads / 32, kMaxCluster = 4, kGradWarps = kGradThreads / 32;
static_assert(kMaxCluster * kGradThreads * kGradCols >= kStepColumns && kMaxGradRows <= kMaxBlockRows, "rows");

// Sums of two values over a row's threads, over the cluster's CTAs too: every warp leaves its share with every CTA, one
// barrier, every warp adds the shares up in the same order.  Two slots by turns: a warp that writes a slot again has passed
// the barrier of the other one, which all warps reach after reading this one.
// (kFirst: the first value is wanted)
template <bool kFirst>
__device__ __forceinline__ float2 exchange(float2 v, float2* share, int cluster, uint32_t rank) {
    if (kFirst) v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int shares = warps * cluster;
    if (shares == 1) return v;
    float2* const row = share + threadIdx.y * shares;
    float2* const at = row + rank * warps + warp;
    if (cluster > 1) {
        if (lane < cluster) {
            const uint32_t dst = mapa_u32(smem_u32(at), lane);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst), "f"(v.x), "f"(v.y) : "memory");
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    } else {
        if (lane == 0) *at = v;
        __syncthreads();
    }
    float2 s = make_float2(0.0f, 0.0f);
    if (shares <= 8) {
        if ((lane & 7) < shares) s = row[lane & 7];
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) {
            if (kFirst) s.x += __shfl_xor_sync(~0u, s.x, o);
            s.y += __shfl_xor_sync(~0u, s.y, o);
        }
        return s;
    }
    for (int i = lane; i < shares; i += 32) {
        const float2 t = row[i];
        s.x += t.x;
        s.y += t.y;
    }
    return make_float2(kFirst ? warp_sum(s.x) : 0.0f, warp_sum(s.y));
}

// A thread's column sums of one vector, in shared memory: 16 bytes of neighbouring threads side by side.
struct ColumnSums {
    uint32_t at, pitch;                      // the thread's first place; bytes of the block's threads' places
    static __device__ __forceinline__ float4 get(uint32_t p) {
        float4 v;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(p) : "memory");
        return v;
    }
    static __device__ __forceinline__ void put(uint32_t p, float4 v) {
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(p), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
    }
    __device__ __forceinline__ void clear() const {
#pragma unroll
        for (int k = 0; k < kGradCols / 4; ++k) put(at + k * pitch, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
    }
    // run c's eight columns: term(j, sum) instead of the j-th pair
    template <typename F>
    __device__ __forceinline__ void add(int c, const F& term) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t p = at + (2 * c + h) * pitch;
            const float4 s = get(p);
            float4 r;
            unpack_f2(term(2 * h, pack_f2(s.x, s.y)), r.x, r.y);
            unpack_f2(term(2 * h + 1, pack_f2(s.z, s.w)), r.z, r.w);
            put(p, r);
        }
    }
};

// kPre, kPost: there is a norm behind / in front of the sum; kMean: one of them subtracts its mean (and has a bias)
template <int kType, bool kPre, bool kPost, bool kMean, bool kWide>
__global__ void __launch_bounds__(kGradThreads, 1)
mip_norm_step_grad_kernel(const __grid_constant__ StepGradArgs a) {
    constexpr bool kAhead = kType != kF32;       // (32-bit elements of two rows do not fit the registers)
    constexpr bool wide = kWide;
    constexpr int kSize = kType == kF32 ? 4 : 2, kRuns = kGradRuns;
    __shared__ alignas(16) uint32_t spread[kWide ? 1 : kGradWarps][kWide ? 4 : (kType == kF32 ? 256 : 128)];
    uint32_t* const buf = spread[kWide ? 0 : (threadIdx.y * blockDim.x + threadIdx.x) >> 5];
    const bool vectors = kWide || a.wide_vectors;
    extern __shared__ float4 sums_smem[];        // column sums: of dpre_w, dpre_b, dpost_w, dpost_b, dgate
    __shared__ float2 share[2][kMaxCluster * kGradWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int cluster = a.cluster;
    const uint32_t rank = cluster > 1 ? cluster_ctarank() : 0u;
    const long long worker = blockIdx.x / static_cast<unsigned>(cluster);
    const int block_rows = blockDim.y, threads = blockDim.x * blockDim.y;
    const long long run = 8ll * blockDim.x;                                // columns between a thread's runs
    const long long col0 = static_cast<long long>(rank) * kRuns * run + 8ll * threadIdx.x;
    int exist[kRuns], warp_exist[kRuns];                 // of the thread's run, of its warp's
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        const long long left = a.N - col0 - c * run;
        exist[c] = left <= 0 ? 0 : (kWide || left >= 8 ? 8 : static_cast<int>(left));
        warp_exist[c] = static_cast<int>(min(max(left + 8 * (threadIdx.x & 31), 0ll), 256ll));
    }
    const Dropout drop(a.mask, a.N);
    const float inv_n = __fdiv_rn(1.0f, static_cast<float>(a.N));
    const bool gate_sum = a.dgate && a.gate_rows > 1, gate_each = a.dgate && a.gate_rows == 1;
    // (vectors that no sum is kept of share the last place)
    int places = 0;
    const auto vector = [&](bool there) {
        const ColumnSums s = {smem_u32(sums_smem) + static_cast<uint32_t>(places * (kGradCols / 4) * threads + threadIdx.y * blockDim.x + threadIdx.x) * 16u,
                              static_cast<uint32_t>(threads) * 16u};
        if (there) {
            s.clear();
            ++places;
        }
        return s;
    };
    const ColumnSums pre_w = vector(kPre), pre_b = vector(kPre && kMean), post_w = vector(kPost), post_b = vector(kPost && kMean), gate_s = vector(gate_sum);

    struct Row {
        Eight<kType> dy[kRuns], dh[kRuns], y[kRuns];
        float4 st;
        bool here;
    };
    const auto at = [&](const void* p, long long row, long long ld) { return static_cast<const char*>(p) + (row * ld + col0) * kSize; };
    const auto load = [&](Row& r, long long base, long long end) {
        const long long row = base + threadIdx.y;
        r.here = row < end;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            const int count = r.here ? exist[c] : 0, limit = r.here ? warp_exist[c] : 0;
            if (a.dY) load_run<kWide>(r.dy[c], at(a.dY, row, a.lddy) + c * run * kSize, count, limit);
            else r.dy[c].clear();
            if (kPre) {
                load_run<kWide>(r.dh[c], at(a.dH, row, a.lddh) + c * run * kSize, count, limit);
                load_run<kWide>(r.y[c], at(a.Y, row, a.ldy) + c * run * kSize, count, limit);
            }
        }
        r.st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if ((kPre || kPost) && r.here) {
            const float* s = a.stats + 4 * row;
            r.st = make_float4(s[0], s[1], s[2], s[3]);
        }
    };
    int slot = 0;
    // (x - mean) * rstd; columns that lie behind the last one are not added up: they are 0
    const auto normalized = [&](uint64_t (&v)[4], float mean, float rstd, int count) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = mul_f2(kMean ? add_f2(v[j], pack_f2(-mean, -mean)) : v[j], pack_f2(rstd, rstd));
        if (kMean || !kWide) clear_behind(v, count);
    };
    // what a norm passes on, but for rstd: g - mean(g) - hat mean(g hat); columns behind the last one stay 0 (the other norm sums over
    // them)
    const auto through = [&](uint64_t (&g)[kRuns][4], const uint64_t (&hat)[kRuns][4], int kind, const int (&count)[kRuns]) {
        uint64_t s = 0ull, u = 0ull;
#pragma unroll
        for (int c = 0; c < kRuns; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (kMean) s = add_f2(s, g[c][j]);
                u = fma_f2(g[c][j], hat[c][j], u);
            }
        slot ^= 1;
        const float2 e = exchange<kMean>(make_float2(kMean ? sum_pair(s) : 0.0f, sum_pair(u)), share[slot], cluster, rank);
        const float mean = kMean && kind == kNormLayer ? -e.x * inv_n : 0.0f, slope = -e.y * inv_n;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            const float m = kWide && count[c] == 0 ? 0.0f : mean;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (kMean) g[c][j] = add_f2(g[c][j], pack_f2(m, m));
                g[c][j] = fma_f2(hat[c][j], pack_f2(slope, slope), g[c][j]);
            }
            if (kMean && !kWide) clear_behind(g[c], count[c]);
        }
    };
    const int gate_kind = a.gate_rows >= a.M ? 0 : (a.gate_rows == 1 ? 1 : 2);       // one row for all, one each, some share one
    const auto process = [&](const Row& r, long long base) {
        const long long row = base + threadIdx.y;
        int count[kRuns], limit[kRuns];
        Eight<kType> z[kRuns], gate[kRuns];
        uint32_t gate_row = gate_kind == 0 || !r.here ? 0u : static_cast<uint32_t>(row);
        if (gate_kind == 2) gate_row /= static_cast<uint32_t>(a.gate_rows);
        uint64_t g[kRuns][4], t[kRuns][4], hat[kRuns][4], w[4];
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            count[c] = r.here ? exist[c] : 0;
            limit[c] = r.here ? warp_exist[c] : 0;
            if (kPost || a.Z) load_run<kWide>(z[c], at(a.Z, row, a.ldz) + c * run * kSize, count[c], limit[c]);
            else z[c].clear();
            if (a.gate) load_run<kWide>(gate[c], at(a.gate, gate_row, a.ldgate) + c * run * kSize, count[c], limit[c]);
        }
        // (drawn here, where the instructions fill the gaps of the first exchange)
        uint4 bits[kRuns];
        if (drop.bar) {
#pragma unroll
            for (int c = 0; c < kRuns; ++c) bits[c] = drop.draw(row, col0 + c * run);
        }
        if (kPre) {
#pragma unroll
            for (int c = 0; c < kRuns; ++c) {
                run_pairs<kWide>(r.dh[c], buf, t[c]);
                run_pairs<kWide>(r.y[c], buf, hat[c]);
                load_vector_pairs(a.pre_w, col0 + c * run, exist[c], vectors, 1.0f, w);
                normalized(hat[c], r.st.z, r.st.w, count[c]);
                pre_w.add(c, [&](int j, uint64_t s) { return fma_f2(t[c][j], hat[c][j], s); });
                if (kMean) pre_b.add(c, [&](int j, uint64_t s) { return add_f2(t[c][j], s); });
#pragma unroll
                for (int j = 0; j < 4; ++j) t[c][j] = mul_f2(t[c][j], w[j]);
            }
            through(t, hat, a.pre, count);
        }
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            run_pairs<kWide>(r.dy[c], buf, g[c]);
            if (kPre) {
#pragma unroll
                for (int j = 0; j < 4; ++j) g[c][j] = fma_f2(t[c][j], pack_f2(r.st.w, r.st.w), g[c][j]);
            }
            if (a.dX) {
                uint64_t x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = mul_f2(pack_f2(a.x_scale, a.x_scale), g[c][j]);
                store_run<kWide, kType>(x, const_cast<char*>(at(a.dX, row, a.lddx)) + c * run * kSize, count[c], limit[c], buf);
            }
            run_pairs<kWide>(z[c], buf, hat[c]);
            if (kPost) {
                load_vector_pairs(a.post_w, col0 + c * run, exist[c], vectors, 1.0f, w);
                normalized(hat[c], r.st.x, r.st.y, count[c]);
            }
            if (!a.gate) {
                if (drop.bar) drop.apply(bits[c], g[c]);
            } else {
                // The mask is taken from the products, not from what is multiplied: 0 times an infinity or a NaN that stands at a dropped
                // place would be a NaN.  Both products in one go share its comparisons (16384 x 4096 bf16, rms norms, gate for each channel
                // 238 us, one by one 246); with a bias behind the block there are no registers for both (layer norms 345, one by one 317).
                constexpr bool kBoth = !(kPost && kMean);
                const uint32_t draws[4] = {bits[c].x, bits[c].y, bits[c].z, bits[c].w};
                uint64_t b[4];
                const auto products = [&](auto masked, auto of_gate, auto of_z) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t k = masked ? drop.scaled(g[c][j]) : g[c][j];
                        const bool lo = !masked || draws[j] << 16 >= drop.bar, hi = !masked || draws[j] >= drop.bar;
                        if (of_gate) {
                            uint64_t u = hat[c][j];
                            if (kPost) u = kMean ? fma_f2(u, w[j], b[j]) : mul_f2(u, w[j]);
                            t[c][j] = mul_f2(k, u);
                            if (masked) t[c][j] = Dropout::where(lo, hi, t[c][j]);
                        }
                        if (of_z) {
                            g[c][j] = mul_f2(k, b[j]);
                            if (masked) g[c][j] = Dropout::where(lo, hi, g[c][j]);
                        }
                    }
                };
                const auto gate_products = [&](auto of_gate, auto of_z) {
                    if (drop.bar) products(std::true_type{}, of_gate, of_z);
                    else products(std::false_type{}, of_gate, of_z);
                };
                if (kBoth) run_pairs<kWide>(gate[c], buf, b);
                if (a.dgate) {
                    if (!kBoth) load_vector_pairs(a.post_b, col0 + c * run, exist[c], vectors, 0.0f, b);
                    gate_products(std::true_type{}, std::bool_constant<kBoth>{});
                    if (gate_each) {
                        store_run<kWide, kType>(t[c], const_cast<char*>(at(a.dgate, row, a.lddgate)) + c * run * kSize, count[c], limit[c], buf);
                    } else {
                        gate_s.add(c, [&](int j, uint64_t s) { return add_f2(t[c][j], s); });
                    }
                }
                if (!kBoth) run_pairs<kWide>(gate[c], buf, b);
                if (!kBoth || !a.dgate) gate_products(std::false_type{}, std::true_type{});
            }
            if (kPost) {
                post_w.add(c, [&](int j, uint64_t s) { return fma_f2(g[c][j], hat[c][j], s); });
                if (kMean) post_b.add(c, [&](int j, uint64_t s) { return add_f2(g[c][j], s); });
#pragma unroll
                for (int j = 0; j < 4; ++j) g[c][j] = mul_f2(g[c][j], w[j]);
            }
        }
        if (kPost) through(g, hat, a.post, count);
        if (a.dZ) {
#pragma unroll
            for (int c = 0; c < kRuns; ++c) {
                if (kPost) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[c][j] = mul_f2(g[c][j], pack_f2(r.st.y, r.st.y));
                }
                store_run<kWide, kType>(g[c], const_cast<char*>(at(a.dZ, row, a.lddz)) + c * run * kSize, count[c], limit[c], buf);
            }
        }
    };
    // A vector's sums over the block's rows, in the first one's threads: eight columns of run c.
    const auto over_block = [&](const ColumnSums& s, int c, float (&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        for (int i = 0; i < block_rows; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 x = ColumnSums::get(s.at + (2 * c + h) * s.pitch + static_cast<uint32_t>(i) * blockDim.x * 16u);
                v[4 * h] += x.x; v[4 * h + 1] += x.y; v[4 * h + 2] += x.z; v[4 * h + 3] += x.w;
            }
        }
    };
    const auto put_sum = [&](const float (&v)[8], float* dst, int c) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < exist[c]) dst[col0 + c * run + j] = v[j];
    };

    // unit u: part u % parts of gate row u / parts (without a gate's sums: of all rows)
    const long long rows_of_gate = gate_sum ? a.gate_rows : a.M;
    const auto unit_rows = [&](long long u, long long& begin, long long& end) {
        const long long g0 = u / a.parts * rows_of_gate, g1 = min(g0 + rows_of_gate, a.M);
        begin = min(g0 + u % a.parts * a.part_rows, g1);
        end = min(begin + a.part_rows, g1);
    };
    if (cluster > 1) {                           // (all CTAs run before anything is sent to one)
        cluster_arrive();
        cluster_wait();
    }
    long long begin, end;
    Row cur;
    if (kAhead && worker < a.units) {
        unit_rows(worker, begin, end);
        load(cur, begin, end);
    }
    for (long long u = worker; u < a.units; u += a.workers) {
        unit_rows(u, begin, end);
        for (long long base = begin; base < end; base += block_rows) {
            if (kAhead) {
                Row next;
                if (base + block_rows < end) {
                    load(next, base + block_rows, end);
                } else if (u + a.workers < a.units) {
                    long long b1, e1;
                    unit_rows(u + a.workers, b1, e1);
                    load(next, b1, e1);
                }
                process(cur, base);
                cur = next;
            } else {
                load(cur, base, end);
                process(cur, base);
            }
        }
        if (kAhead && begin >= end && u + a.workers < a.units) {     // (a part without rows: nothing has been loaded for the next)
            long long b1, e1;
            unit_rows(u + a.workers, b1, e1);
            load(cur, b1, e1);
        }
        if (gate_sum) {
            if (block_rows > 1) __syncthreads();
            if (threadIdx.y == 0) {
#pragma unroll
                for (int c = 0; c < kRuns; ++c) {
                    float v[8];
                    over_block(gate_s, c, v);
                    if (a.parts > 1) {
                        put_sum(v, a.gate_part + u * a.N, c);
                    } else {
                        Eight<kType> e;
                        e.set(v);
                        e.store(a.dgate, u * a.lddgate + col0 + c * run, exist[c], wide);
                    }
                }
            }
            if (block_rows > 1) __syncthreads();
            gate_s.clear();
        }
    }
    if (a.sums == 0) return;
    if (block_rows > 1) __syncthreads();
    if (threadIdx.y != 0) return;
    float* plane = a.sum_part + worker * a.sums * a.N;
    const auto put = [&](const ColumnSums& s, const float* wanted) {
        if (!wanted) return;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            float v[8];
            over_block(s, c, v);
            put_sum(v, plane, c);
        }
        plane += a.N;
    };
    if (kPost) {
        put(post_w, a.dpost_w);
        if (kMean) put(post_b, a.dpost_b);
    }
    if (kPre) {
        put(pre_w, a.dpre_w);
        if (kMean) put(pre_b, a.dpre_b);
    }
}

// Column sums of planes: job j < sums adds the workers' planes of one vector, the others the parts of one row of dgate.
// 32 columns a block, 16 rows of threads take every 16th plane, then one adds the 16.
constexpr int kSumRows = 16;
struct SumArgs {
    long long N, workers, parts, groups;
    int sums, type;
    const float* sum_part;
    const float* gate_part;
    float* out[4];
    void* dgate; long long lddgate;
};
__global__ void __launch_bounds__(32 * kSumRows)
mip_norm_step_sums_kernel(const SumArgs a) {
    __shared__ float share[kSumRows][32];
    const long long job = blockIdx.y, col = 32ll * blockIdx.x + threadIdx.x;
    const bool vec = job < a.sums;
    const long long planes = vec ? a.workers : a.parts, pitch = vec ? a.sums * a.N : a.N;
    const float* src = vec ? a.sum_part + job * a.N : a.gate_part + (job - a.sums) * a.parts * a.N;
    float s = 0.0f;
    if (col < a.N) {
#pragma unroll 4
        for (long long p = threadIdx.y; p < planes; p += kSumRows) s += src[p * pitch + col];
    }
    share[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y != 0 || col >= a.N) return;
#pragma unroll
    for (int i = 1; i < kSumRows; ++i) s += share[i][threadIdx.x];
    if (vec) a.out[job][col] = s;
    else store_element(a.dgate, (job - a.sums) * a.lddgate + col, a.type, s);
}

// More shared memory than a kernel has without asking is asked for once per kernel and device, at its first launch there (which
// loads it: that does not belong to a graph being captured).
constexpr int kMostSums = 5 * kGradCols * 4 * kGradThreads;
template <typename Kernel>
cudaError_t grad_launch(Kernel kernel, std::atomic<unsigned long long>& asked, const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(asked.load(std::memory_order_acquire) & bit)) {
        cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
        (void)cudaThreadExchangeStreamCaptureMode(&mode);
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSums);
        (void)cudaThreadExchangeStreamCaptureMode(&mode);
        if (e != cudaSuccess) return e;
        asked.fetch_or(bit, std::memory_order_release);
    }
    return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <int kType, bool kPre, bool kPost, bool kMean, bool kWide>
cudaError_t grad_one(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    static std::atomic<unsigned long long> asked{0};
    return grad_launch(mip_norm_step_grad_kernel<kType, kPre, kPost, kMean, kWide>, asked, a, cfg);
}
template <int kType, bool kPre, bool kPost, bool kWide>
cudaError_t grad_mean(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    if ((kPre && a.pre == kNormLayer) || (kPost && a.post == kNormLayer)) {
        if constexpr (kPre || kPost) return grad_one<kType, kPre, kPost, true, kWide>(a, cfg);
    }
    return grad_one<kType, kPre, kPost, false, kWide>(a, cfg);
}
template <int kType, bool kWide>
cudaError_t grad_t(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    if (a.pre != kNormNone) return a.post != kNormNone ? grad_mean<kType, true, true, kWide>(a, cfg) : grad_mean<kType, true, false, kWide>(a, cfg);
    return a.post != kNormNone ? grad_mean<kType, false, true, kWide>(a, cfg) : grad_mean<kType, false, false, kWide>(a, cfg);
}
template <int kType>
cudaError_t grad_wide(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    return a.wide ? grad_t<kType, true>(a, cfg) : grad_t<kType, false>(a, cfg);
}

struct GradShape {
    int cluster, threads, rows;
};
GradShape grad_shape(long long N) {
    GradShape s;
    s.cluster = static_cast<int>((N + kGradCols * kGradThreads - 1) / (kGradCols * kGradThreads));
    s.threads = static_cast<int>(((N + kGradCols * s.cluster - 1) / (kGradCols * s.cluster) + 31) / 32 * 32);
    s.rows = s.threads >= kBlockThreads ? 1 : kBlockThreads / s.threads;
    return s;
}
size_t sums_bytes(const StepGradArgs& a, const GradShape& s) {
    const bool mean = a.pre == kNormLayer || a.post == kNormLayer;
    const int per_norm = mean ? 2 : 1;
    const int vectors = (a.pre != kNormNone ? per_norm : 0) + (a.post != kNormNone ? per_norm : 0) + (a.dgate && a.gate_rows > 1 ? 1 : 0);
    return static_cast<size_t>(vectors) * kGradCols * 4 * s.threads * s.rows;
}

}  // namespace

// How the rows are dealt: fills a's cluster, workers, units, parts and part_rows; returns the scratch bytes needed: no more than
// `per_sm` planes of N float32 for each SM and vector.
size_t plan_norm_step_grad(StepGradArgs& a, int sm_count, int per_sm) {
    const GradShape s = grad_shape(a.N);
    a.cluster = s.cluster;
    // (512 threads of up to 128 registers fill an SM, and their sums' shared memory: 160 KB at most; three CTAs are those of rows of 2049
    // to 2560 columns: with two 16384 x 2560 bf16 156 -> 192 us)
    const int here = std::min(per_sm, kGradThreads / (s.threads * s.rows));
    const long long resident = std::max<long long>(1, static_cast<long long>(sm_count) * here / s.cluster);
    const bool gate_sum = a.dgate && a.gate_rows > 1;
    const long long group_rows = gate_sum ? std::min(a.gate_rows, a.M) : a.M;
    const long long groups = (a.M + group_rows - 1) / group_rows;
    const long long most = (group_rows + s.rows - 1) / s.rows;                     // parts of a group that have rows
    a.parts = std::max<long long>(1, std::min(most, resident / groups));
    a.part_rows = (group_rows + a.parts - 1) / a.parts;
    a.part_rows = (a.part_rows + s.rows - 1) / s.rows * s.rows;
    a.parts = (group_rows + a.part_rows - 1) / a.part_rows;
    a.units = groups * a.parts;
    a.workers = std::min(a.units, resident);
    const size_t sums = static_cast<size_t>(a.workers) * a.sums * a.N * 4, gate = gate_sum && a.parts > 1 ? static_cast<size_t>(a.units) * a.N * 4 : 0;
    return sums + gate;
}

cudaError_t launch_norm_step_grad(int type, StepGradArgs a, void* scratch, cudaStream_t stream, int* launches) {
    const GradShape s = grad_shape(a.N);
    a.sum_part = static_cast<float*>(scratch);
    a.gate_part = a.sum_part + a.workers * a.sums * a.N;
    const bool gate_sum = a.dgate && a.gate_rows > 1;
    if (a.M > 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(a.workers * s.cluster));
        cfg.blockDim = dim3(static_cast<unsigned>(s.threads), static_cast<unsigned>(s.rows));
        cfg.dynamicSmemBytes = sums_bytes(a, s);
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = static_cast<unsigned>(s.cluster);
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = pdl_allowed();
        cfg.attrs = s.cluster > 1 ? attr : attr + 1;
        cfg.numAttrs = s.cluster > 1 ? 1 : (cfg.gridDim.x <= 128 ? 1 : 0);
        const cudaError_t e = type == kF32 ? grad_wide<kF32>(a, cfg) : (type == kF16 ? grad_wide<kF16>(a, cfg) : grad_wide<kBF16>(a, cfg));
        ++*launches;
        if (e != cudaSuccess) return e;
    }
    const bool gate_parts = gate_sum && a.parts > 1;
    if (a.sums == 0 && !gate_parts) return cudaSuccess;
    SumArgs f = {};
    f.N = a.N;
    f.workers = a.M > 0 ? a.workers : 0;
    f.parts = a.parts;
    f.groups = gate_parts ? a.units / a.parts : 0;
    f.sums = a.sums;
    f.type = type;
    f.sum_part = a.sum_part;
    f.gate_part = a.gate_part;
    f.dgate = a.dgate;
    f.lddgate = a.lddgate;
    int at = 0;
    for (float* p : {a.dpost_w, a.dpost_b, a.dpre_w, a.dpre_b})
        if (p) f.out[at++] = p;
    const dim3 grid(static_cast<unsigned>((a.N + 31) / 32), static_cast<unsigned>(a.sums + f.groups));
    mip_norm_step_sums_kernel<<<grid, dim3(32, kSumRows), 0, stream>>>(f);
    ++*launches;
    return cudaGetLastError();
}

}  // namespace mip
