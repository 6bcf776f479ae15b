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
__device__ __forceinline__ float2 exchange(float2 v, RowExchange& x, int slot, int cluster, uint32_t rank) {
    v.x = warp_sum(v.x);
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
    float2 s = make_float2(0.0f, 0.0f);
    for (int i = lane; i < shares; i += 32) {
        const float2 t = x.share[slot][threadIdx.y][i];
        s.x += t.x;
        s.y += t.y;
    }
    return make_float2(warp_sum(s.x), warp_sum(s.y));
}

// kPre, kPost: there is a norm behind / in front of the sum; kMean: one of them subtracts its mean (and has a bias)
template <int kType, bool kPre, bool kPost, bool kMean>
__global__ void __launch_bounds__(kGradThreads, 1)
mip_norm_step_grad_kernel(const StepGradArgs a) {
    constexpr bool kAhead = kType != kF32;       // (32-bit elements of two rows leave no registers for the sums)
    __shared__ RowExchange ex;
    __shared__ float rows_sum[kMaxGradRows - 1][8 * 64];
    pdl_wait();
    pdl_launch_dependents();
    const int cluster = a.cluster;
    const uint32_t rank = cluster > 1 ? cluster_ctarank() : 0u;
    const long long worker = blockIdx.x / static_cast<unsigned>(cluster);
    const int block_rows = blockDim.y;
    const bool wide = a.wide;
    const long long col = 8ll * (static_cast<long long>(rank) * blockDim.x + threadIdx.x);
    const int exist = a.N <= col ? 0 : (a.N - col < 8 ? static_cast<int>(a.N - col) : 8);
    const Dropout drop = dropout_of(a.bar, a.drop_scale, a.seed, a.counter, a.N);
    const float inv_n = __fdiv_rn(1.0f, static_cast<float>(a.N));
    const bool gate_sum = a.dgate && a.gate_rows > 1, gate_each = a.dgate && a.gate_rows == 1;
    float pre_w[8] = {}, pre_b[8] = {}, post_w[8] = {}, post_b[8] = {}, gate_s[8] = {};

    struct Row {
        Eight<kType> dy, dh, y, z;
        float4 st;
        int count;
    };
    const auto load = [&](Row& r, long long base, long long end) {
        const long long row = base + threadIdx.y;
        const bool here = row < end;
        r.count = here ? exist : 0;
        if (a.dY) r.dy.load(a.dY, row * a.lddy + col, r.count, wide);
        else r.dy.clear();
        if (kPre) {
            r.dh.load(a.dH, row * a.lddh + col, r.count, wide);
            r.y.load(a.Y, row * a.ldy + col, r.count, wide);
        }
        if (kPost || a.Z) r.z.load(a.Z, row * a.ldz + col, r.count, wide);
        else r.z.clear();
        r.st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if ((kPre || kPost) && here) {
            const float* s = a.stats + 4 * row;
            r.st = make_float4(s[0], s[1], s[2], s[3]);
        }
    };
    // (columns that lie behind the last one are not added up: their y^ may be anything)
    int slot = 0;
    const auto process = [&](const Row& r, long long base) {
        const long long row = base + threadIdx.y;
        float g[8], t[8], w[8];
        r.dy.values(g);
        if (kPre) {
            float hat[8];
            r.dh.values(t);
            r.y.values(hat);
            load_vector8(a.pre_w, col, exist, wide, 1.0f, w);
            float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hat[j] = j < r.count ? (hat[j] - r.st.z) * r.st.w : 0.0f;
                pre_w[j] = fmaf(t[j], hat[j], pre_w[j]);
                if (kMean) pre_b[j] += t[j];
                t[j] *= w[j];
                if (kMean) s.x += t[j];
                s.y = fmaf(t[j], hat[j], s.y);
            }
            s = exchange(s, ex, slot ^= 1, cluster, rank);
            const float mean = kMean && a.pre == kNormLayer ? s.x * inv_n : 0.0f, slope = s.y * inv_n;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = fmaf(t[j] - mean - hat[j] * slope, r.st.w, g[j]);
        }
        if (a.dX) {
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = a.x_scale * g[j];
            Eight<kType> e;
            e.set(t);
            e.store(a.dX, row * a.lddx + col, r.count, wide);
        }
        if (drop.bar) {
            uint64_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = pack_f2(g[2 * j], g[2 * j + 1]);
            drop.apply(drop.draw(row, col), u);
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack_f2(u[j], g[2 * j], g[2 * j + 1]);
        }
        float hat[8];
        r.z.values(hat);
        if (kPost) {
            load_vector8(a.post_w, col, exist, wide, 1.0f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) hat[j] = j < r.count ? (hat[j] - r.st.x) * r.st.y : 0.0f;
        }
        if (a.gate) {
            if (a.dgate) {
                float b[8];
                if (kPost) load_vector8(a.post_b, col, exist, wide, 0.0f, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = g[j] * (kPost ? fmaf(hat[j], w[j], b[j]) : hat[j]);
                if (gate_each) {
                    Eight<kType> e;
                    e.set(t);
                    e.store(a.dgate, row * a.lddgate + col, r.count, wide);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) gate_s[j] += t[j];
                }
            }
            Eight<kType> e;
            e.load(a.gate, (r.count ? static_cast<uint32_t>(row) / static_cast<uint32_t>(a.gate_rows) : 0u) * a.ldgate + col, r.count, wide);
            e.values(t);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] *= t[j];
        }
        if (kPost) {
            float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                post_w[j] = fmaf(g[j], hat[j], post_w[j]);
                if (kMean) post_b[j] += g[j];
                g[j] *= w[j];
                if (kMean) s.x += g[j];
                s.y = fmaf(g[j], hat[j], s.y);
            }
            s = exchange(s, ex, slot ^= 1, cluster, rank);
            const float mean = kMean && a.post == kNormLayer ? s.x * inv_n : 0.0f, slope = s.y * inv_n;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = (g[j] - mean - hat[j] * slope) * r.st.y;
        }
        if (a.dZ) {
            Eight<kType> e;
            e.set(g);
            e.store(a.dZ, row * a.lddz + col, r.count, wide);
        }
    };
    // Adds the block's rows' sums up in the first one's registers.
    const auto over_block = [&](float (&v)[8]) {
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
            over_block(gate_s);
            if (a.parts > 1) {
                put_sum(gate_s, a.gate_part + u * a.N);
            } else if (threadIdx.y == 0) {
                Eight<kType> e;
                e.set(gate_s);
                e.store(a.dgate, u * a.lddgate + col, exist, wide);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) gate_s[j] = 0.0f;
        }
    }
    if (a.sums == 0) return;
    float* plane = a.sum_part + worker * a.sums * a.N;
    int at = 0;
    const auto put = [&](float (&v)[8], const float* wanted) {
        if (!wanted) return;
        over_block(v);
        put_sum(v, plane + at * a.N);
        ++at;
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

template <int kType, bool kPre, bool kPost>
cudaError_t grad_mean(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    if ((kPre && a.pre == kNormLayer) || (kPost && a.post == kNormLayer)) {
        if constexpr (kPre || kPost) return cudaLaunchKernelEx(&cfg, mip_norm_step_grad_kernel<kType, kPre, kPost, true>, a);
    }
    return cudaLaunchKernelEx(&cfg, mip_norm_step_grad_kernel<kType, kPre, kPost, false>, a);
}
template <int kType>
cudaError_t grad_t(const StepGradArgs& a, const cudaLaunchConfig_t& cfg) {
    if (a.pre != kNormNone) return a.post != kNormNone ? grad_mean<kType, true, true>(a, cfg) : grad_mean<kType, true, false>(a, cfg);
    return a.post != kNormNone ? grad_mean<kType, false, true>(a, cfg) : grad_mean<kType, false, false>(a, cfg);
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
        const cudaError_t e = type == kF32 ? grad_t<kF32>(a, cfg) : (type == kF16 ? grad_t<kF16>(a, cfg) : grad_t<kBF16>(a, cfg));
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
