// The step between two blocks of a transformer layer, backward: from the gradients of y and h those of x, z, the gate and
// the norms' weights and biases.  With ^ for a normalised value and q, p for the reciprocal deviations of the two norms:
//     g = dy + q (w dh - mean(w dh) - y^ mean(w dh y^)),   dx = s g,
//     k = mask g,   dgate = sum k u,   m = gate k,   dz = p (w' m - mean(w' m) - z^ mean(w' m z^))
// (the first means for a norm that subtracts its mean only), and over all rows dw = sum dh y^, db = sum dh,
// dw' = sum m z^, db' = sum m.  The rows' statistics come from the forward pass, so each norm needs one exchange; the mask
// is drawn again from its counter.
//
// Workers (CTAs, or clusters of CTAs that share a row of more than 4096 columns) go through the rows and keep the column sums in
// registers, eight columns a thread; a second kernel adds the workers' sums in a fixed order.  Rows are dealt in units that
// lie within one gate row, so that a unit's sum is a share of one row of dgate.  While a row waits for its exchanges, the next
// one's elements are on their way.
//
// What bounds it: the bytes of dy, dh, y, z, dx and dz.
#include <algorithm>

#include "ptx.cuh"
#include "step_math.cuh"

namespace mip {

namespace {

constexpr int kMaxGradRows = 4, kMaxCluster = 8, kGradThreads = 512, kGradWarps = kGradThreads / 32;

// Sums of two values over a row's threads, over the cluster's CTAs too: every warp leaves its share with every CTA, one
// barrier, every warp adds the shares up in the same order.  Two slots by turns: a warp that writes a slot again has passed
// the barrier of the other one, which all warps reach after reading this one.
struct RowExchange {
    float2 share[2][kMaxGradRows][kMaxCluster * kGradWarps];
};
// (kFirst: the first value is wanted)
template <bool kFirst>
__device__ __forceinline__ float2 exchange(float2 v, RowExchange& x, int slot, int cluster, uint32_t rank) {
    if (kFirst) v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int shares = warps * cluster;
    if (shares == 1) return v;
    float2* at = &x.share[slot][threadIdx.y][rank * warps + warp];
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
    if (shares <= kGradWarps) {
        const int i = lane & (kGradWarps - 1);
        float2 s = i < shares ? x.share[slot][threadIdx.y][i] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int o = kGradWarps / 2; o > 0; o >>= 1) {
            if (kFirst) s.x += __shfl_xor_sync(~0u, s.x, o);
            s.y += __shfl_xor_sync(~0u, s.y, o);
        }
        return s;
    }
    float2 s = make_float2(0.0f, 0.0f);
    for (int i = lane; i < shares; i += 32) {
        const float2 t = x.share[slot][threadIdx.y][i];
        s.x += t.x;
        s.y += t.y;
    }
    return make_float2(warp_sum(s.x), warp_sum(s.y));
}

// kPre, kPost: there is a norm behind / in front of the sum; kMean: one of them subtracts its mean (and has a bias)
template <int kType, bool kPre, bool kPost, bool kMean, bool kWide>
__global__ void __launch_bounds__(kGradThreads, 1)
mip_norm_step_grad_kernel(const StepGradArgs a) {
    constexpr bool kAhead = kType != kF32;       // (32-bit elements of two rows leave no registers for the sums)
    constexpr bool wide = kWide;
    constexpr int kSize = kType == kF32 ? 4 : 2;
    __shared__ RowExchange ex;
    __shared__ float rows_sum[kMaxGradRows - 1][8 * 64];
    pdl_wait();
    pdl_launch_dependents();
    const int cluster = a.cluster;
    const uint32_t rank = cluster > 1 ? cluster_ctarank() : 0u;
    const long long worker = blockIdx.x / static_cast<unsigned>(cluster);
    const int block_rows = blockDim.y;
    const long long col = 8ll * (static_cast<long long>(rank) * blockDim.x + threadIdx.x);
    const int exist = a.N <= col ? 0 : (a.N - col < 8 ? static_cast<int>(a.N - col) : 8);
    const Dropout drop = dropout_of(a.bar, a.drop_scale, a.seed, a.counter, a.N);
    const float inv_n = __fdiv_rn(1.0f, static_cast<float>(a.N));
    const bool gate_sum = a.dgate && a.gate_rows > 1, gate_each = a.dgate && a.gate_rows == 1;
    uint64_t pre_w[4] = {}, pre_b[4] = {}, post_w[4] = {}, post_b[4] = {}, gate_s[4] = {};      // sums

    struct Row {
        Eight<kType> dy, dh, y, z;
        float4 st;
        int count;
    };
    const auto at = [&](const void* p, long long row, long long ld) { return static_cast<const char*>(p) + (row * ld + col) * kSize; };
    const auto load = [&](Row& r, long long base, long long end) {
        const long long row = base + threadIdx.y;
        const bool here = row < end;
        r.count = here ? exist : 0;
        if (a.dY) r.dy.load(at(a.dY, row, a.lddy), 0, r.count, wide);
        else r.dy.clear();
        if (kPre) {
            r.dh.load(at(a.dH, row, a.lddh), 0, r.count, wide);
            r.y.load(at(a.Y, row, a.ldy), 0, r.count, wide);
        }
        if (kPost || a.Z) r.z.load(at(a.Z, row, a.ldz), 0, r.count, wide);
        else r.z.clear();
        r.st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if ((kPre || kPost) && here) {
            const float* s = a.stats + 4 * row;
            r.st = make_float4(s[0], s[1], s[2], s[3]);
        }
    };
    Eight<kType> gate;
    uint32_t gate_row = ~0u;
    int slot = 0;
    // (x - mean) * rstd; columns that lie behind the last one are not added up: they are 0
    const auto normalized = [&](uint64_t (&v)[4], float mean, float rstd, int count) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = mul_f2(kMean ? add_f2(v[j], pack_f2(-mean, -mean)) : v[j], pack_f2(rstd, rstd));
        if (kMean || !kWide) clear_behind(v, count);
    };
    // sums over the row of g and g hat, and what a norm passes on: rstd (g - mean(g) - hat mean(g hat))
    const auto through = [&](uint64_t (&g)[4], const uint64_t (&hat)[4], int kind, float rstd, const auto& take) {
        uint64_t s = 0ull, u = 0ull;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (kMean) s = add_f2(s, g[j]);
            u = fma_f2(g[j], hat[j], u);
        }
        const float2 e = exchange<kMean>(make_float2(kMean ? sum_pair(s) : 0.0f, sum_pair(u)), ex, slot ^= 1, cluster, rank);
        const float mean = kMean && kind == kNormLayer ? -e.x * inv_n : 0.0f, slope = -e.y * inv_n;
#pragma unroll
        for (int j = 0; j < 4; ++j) take(j, fma_f2(hat[j], pack_f2(slope, slope), kMean ? add_f2(g[j], pack_f2(mean, mean)) : g[j]), pack_f2(rstd, rstd));
    };
    const auto process = [&](const Row& r, long long base) {
        const long long row = base + threadIdx.y;
        if (a.gate && r.count) {                             // (read again where the row has another gate row than the last one)
            const uint32_t i = a.gate_rows == 1 ? static_cast<uint32_t>(row)
                               : (a.gate_rows >= a.M ? 0u : static_cast<uint32_t>(row) / static_cast<uint32_t>(a.gate_rows));
            if (i != gate_row) gate.load(a.gate, i * a.ldgate + col, exist, wide);
            gate_row = i;
        }
        uint64_t g[4], t[4], w[4];
        r.dy.pairs(g);
        if (kPre) {
            uint64_t hat[4];
            r.dh.pairs(t);
            r.y.pairs(hat);
            load_vector_pairs(a.pre_w, col, exist, wide, 1.0f, w);
            normalized(hat, r.st.z, r.st.w, r.count);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pre_w[j] = fma_f2(t[j], hat[j], pre_w[j]);
                if (kMean) pre_b[j] = add_f2(pre_b[j], t[j]);
                t[j] = mul_f2(t[j], w[j]);
            }
            through(t, hat, a.pre, r.st.w, [&](int j, uint64_t v, uint64_t rstd) { g[j] = fma_f2(v, rstd, g[j]); });
        }
        if (a.dX) {
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = mul_f2(pack_f2(a.x_scale, a.x_scale), g[j]);
            Eight<kType> e;
            e.set_pairs(t);
            e.store(const_cast<char*>(at(a.dX, row, a.lddx)), 0, r.count, wide);
        }
        if (drop.bar) drop.apply(drop.draw(row, col), g);
        uint64_t hat[4];
        r.z.pairs(hat);
        if (kPost) {
            load_vector_pairs(a.post_w, col, exist, wide, 1.0f, w);
            normalized(hat, r.st.x, r.st.y, r.count);
        }
        if (a.gate) {
            if (a.dgate) {
                uint64_t b[4];
                if (kPost && kMean) load_vector_pairs(a.post_b, col, exist, wide, 0.0f, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint64_t u = hat[j];
                    if (kPost) u = kMean ? fma_f2(u, w[j], b[j]) : mul_f2(u, w[j]);
                    t[j] = mul_f2(g[j], u);
                }
                if (gate_each) {
                    Eight<kType> e;
                    e.set_pairs(t);
                    e.store(a.dgate, row * a.lddgate + col, r.count, wide);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) gate_s[j] = add_f2(gate_s[j], t[j]);
                }
            }
            if (r.count) {
                gate.pairs(t);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = mul_f2(g[j], t[j]);
            }
        }
        if (kPost) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                post_w[j] = fma_f2(g[j], hat[j], post_w[j]);
                if (kMean) post_b[j] = add_f2(post_b[j], g[j]);
                g[j] = mul_f2(g[j], w[j]);
            }
            through(g, hat, a.post, r.st.y, [&](int j, uint64_t v, uint64_t rstd) { g[j] = mul_f2(v, rstd); });
        }
        if (a.dZ) {
            Eight<kType> e;
            e.set_pairs(g);
            e.store(const_cast<char*>(at(a.dZ, row, a.lddz)), 0, r.count, wide);
        }
    };
    // Adds the block's rows' sums up in the first one's registers.
    const auto over_block = [&](const uint64_t (&pairs)[4], float (&v)[8]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack_f2(pairs[j], v[2 * j], v[2 * j + 1]);
        if (block_rows == 1) return;
        if (threadIdx.y > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) rows_sum[threadIdx.y - 1][8 * threadIdx.x + j] = v[j];
        }
        __syncthreads();
        if (threadIdx.y == 0) {
            for (int i = 0; i < block_rows - 1; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += rows_sum[i][8 * threadIdx.x + j];
        }
        __syncthreads();
    };
    const auto put_sum = [&](const float (&v)[8], float* dst) {
        if (threadIdx.y != 0) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < exist) dst[col + j] = v[j];
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
    if (worker < a.units) {
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
            float v[8];
            over_block(gate_s, v);
            if (a.parts > 1) {
                put_sum(v, a.gate_part + u * a.N);
            } else if (threadIdx.y == 0) {
                Eight<kType> e;
                e.set(v);
                e.store(a.dgate, u * a.lddgate + col, exist, wide);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) gate_s[j] = 0ull;
        }
    }
    if (a.sums == 0) return;
    float* plane = a.sum_part + worker * a.sums * a.N;
    int place = 0;
    const auto put = [&](const uint64_t (&pairs)[4], const float* wanted) {
        if (!wanted) return;
        float v[8];
        over_block(pairs, v);
        put_sum(v, plane + place * a.N);
        ++place;
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

template <int kType, bool kPre, bool kPost, bool kWide>
cudaError_t grad_mean(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    if ((kPre && a.pre == kNormLayer) || (kPost && a.post == kNormLayer)) {
        if constexpr (kPre || kPost) return cudaLaunchKernelEx(&cfg, mip_norm_step_grad_kernel<kType, kPre, kPost, true, kWide>, a);
    }
    return cudaLaunchKernelEx(&cfg, mip_norm_step_grad_kernel<kType, kPre, kPost, false, kWide>, a);
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
    s.cluster = static_cast<int>((N + 8 * kGradThreads - 1) / (8 * kGradThreads));
    s.threads = static_cast<int>(((N + 8 * s.cluster - 1) / (8 * s.cluster) + 31) / 32 * 32);
    s.rows = s.threads >= 128 ? 1 : 128 / s.threads;             // (up to kMaxGradRows)
    return s;
}

}  // namespace

// How the rows are dealt: fills a's cluster, workers, units, parts and part_rows; returns the scratch bytes needed.
size_t plan_norm_step_grad(StepGradArgs& a, int sm_count) {
    const GradShape s = grad_shape(a.N);
    a.cluster = s.cluster;
    // (512 threads of up to 128 registers fill an SM)
    const long long resident = std::max<long long>(1, static_cast<long long>(sm_count) * (kGradThreads / (s.threads * s.rows)) / s.cluster);
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
