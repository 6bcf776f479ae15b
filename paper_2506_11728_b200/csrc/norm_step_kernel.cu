// The step between two blocks of a transformer layer, forward:
//     v = dropout(gate * norm_post(z)),  y = s x + v,  h = norm_pre(y),  h as values and/or as 8-bit codes,
// every part optional.  Two norms, a gate, a mask, the residual sum and the codes in one pass: x and z are read once, y and h
// (or h's codes) written once, and the mask exists nowhere but in registers.
//
// A row stays in the registers of its threads, runs of eight neighbouring columns each (rows of up to 32768 columns).  Means
// come first, then the squares of what is left, so that a large mean takes no digits from the variance.  The dropout mask is a
// function of (seed, counter, row, column): one draw of a counter-based generator for eight columns.
//
// What bounds it: the bytes of x, z, y and h, and close behind them the instructions (two norms, a gate and the generator's ten
// rounds on every eight columns).  Hence packed arithmetic on pairs, 16 columns a thread (a row's exchanges cost a warp the same
// whatever it holds), blocks that go on from row to row with the norms' weights in registers, and the next row's elements on
// their way while a row waits for its exchanges.  With few rows each gets a block of its own and eight columns a thread.
//
// Measured, 16384 x 4096 bf16: two norms, a gate for each channel and dropout 132 us, without dropout 105 (the bytes: 82), x and z to y
// and codes 92 (72); without norms, with dropout 76, without 68.  Rows at no 16-byte boundary (a row's 256 columns by turns of a
// warp's lanes, then through shared memory) take 1.4 (f32) to 2.3 times (16 bits) as long.
#include <algorithm>

#include "ptx.cuh"
#include "step_math.cuh"

namespace mip {

namespace {

// Sum over a row's threads; all of them get it.  Two exchange buffers by turns: who writes one again has passed the barrier of
// the other, which all reach after reading this one.
template <int kThreads>
struct Exchange {
    float part[2][kMaxBlockRows][kThreads / 32];
};
template <int kThreads, typename F>
__device__ __forceinline__ float over_warps(float v, Exchange<kThreads>& x, int& slot, const F& join) {
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    slot ^= 1;
    constexpr int kMost = kThreads / 32;
    if ((threadIdx.x & 31) == 0) x.part[slot][threadIdx.y][threadIdx.x >> 5] = v;
    __syncthreads();
    const int i = threadIdx.x & (kMost - 1);
    v = i < warps ? x.part[slot][threadIdx.y][i] : 0.0f;
#pragma unroll
    for (int o = kMost / 2; o > 0; o >>= 1) v = join(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
template <int kThreads>
__device__ __forceinline__ float row_sum(float v, Exchange<kThreads>& x, int& slot) {
    return over_warps(warp_sum(v), x, slot, [](float a, float b) { return a + b; });
}
// (bits of magnitudes, 0 and up: they order like integers)
template <int kThreads>
__device__ __forceinline__ uint32_t row_max(uint32_t v, Exchange<kThreads>& x, int& slot) {
    return __float_as_uint(over_warps(__uint_as_float(__reduce_max_sync(~0u, v)), x, slot,
                                      [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
}

// v becomes (v - mean) / sqrt(var + eps); returns (mean, 1 / sqrt(var + eps)).
template <int kRuns, int kThreads>
__device__ __forceinline__ float2 normalize(int kind, uint64_t (&v)[kRuns][4], const int (&count)[kRuns], float inv_n, float eps, Exchange<kThreads>& x, int& slot) {
    float mean = 0.0f;
    if (kind == kNormLayer) {
        uint64_t s = 0ull;
#pragma unroll
        for (int c = 0; c < kRuns; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) s = add_f2(s, v[c][j]);        // (columns that do not exist hold 0)
        mean = row_sum(sum_pair(s), x, slot) * inv_n;
        const uint64_t m = pack_f2(-mean, -mean);
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[c][j] = add_f2(v[c][j], m);
            clear_behind(v[c], count[c]);
        }
    }
    uint64_t q = 0ull;
#pragma unroll
    for (int c = 0; c < kRuns; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) q = fma_f2(v[c][j], v[c][j], q);
    const float rstd = rsqrtf(fmaf(row_sum(sum_pair(q), x, slot), inv_n, eps));
#pragma unroll
    for (int c = 0; c < kRuns; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[c][j] = mul_f2(v[c][j], pack_f2(rstd, rstd));
    return make_float2(mean, rstd);
}
// v w + b; w (the row's own copy, or read again) and b as they are wanted
template <int kRuns>
__device__ __forceinline__ void affine(uint64_t (&v)[kRuns][4], const uint64_t (&kept)[kRuns][4], bool keep, const float* w, const float* b,
                                       const long long (&col)[kRuns], const int (&exist)[kRuns], bool wide) {
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        if (w) {
            uint64_t x[4];
            if (!keep) load_vector_pairs(w, col[c], exist[c], wide, 1.0f, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[c][j] = mul_f2(v[c][j], keep ? kept[c][j] : x[j]);
        }
        if (b) {
            uint64_t x[4];
            load_vector_pairs(b, col[c], exist[c], wide, 0.0f, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[c][j] = add_f2(v[c][j], x[j]);
        }
    }
}

__device__ __forceinline__ void store_codes8(uint8_t* dst, uint2 q, int count, bool wide) {
    if (wide) {
        if (count > 0) *reinterpret_cast<uint2*>(dst) = q;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) dst[j] = static_cast<uint8_t>((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
    }
}

// kRuns runs of eight columns a thread, up to kThreads threads a block; kAhead: a row's elements are asked for while the one before
// is worked on, and the norms' weights are kept.  kPost, kPre: there may be such a norm; without any, registers are few, and many
// blocks on an SM do what reading ahead does.
template <int kType, int kRuns, int kThreads, bool kAhead, bool kWide, bool kPost, bool kPre>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? (kPost || kPre ? 2 : (kWide || kType != kF32 ? 4 : 3)) : 1)
mip_norm_step_kernel(const __grid_constant__ StepArgs a) {
    __shared__ Exchange<kThreads> ex;
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool wide = kWide;
    __shared__ alignas(16) uint32_t spread[kWide ? 1 : kThreads / 32][kWide ? 4 : (kType == kF32 ? 256 : 128)];
    uint32_t* const buf = spread[kWide ? 0 : (threadIdx.y * blockDim.x + threadIdx.x) >> 5];
    const bool vectors = kWide || a.wide_vectors;
    const Dropout drop(a.mask, a.N);
    const float inv_n = __fdiv_rn(1.0f, static_cast<float>(a.N));
    int slot = 0;
    long long col[kRuns];
    int exist[kRuns], warp_exist[kRuns];                 // of the thread's run, of its warp's
    uint64_t post_w[kRuns][4], pre_w[kRuns][4];
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        col[c] = 8ll * ((static_cast<long long>(blockIdx.y) * kRuns + c) * blockDim.x + threadIdx.x);
        const long long left = a.N - col[c];
        exist[c] = left <= 0 ? 0 : (kWide || left >= 8 ? 8 : static_cast<int>(left));
        warp_exist[c] = static_cast<int>(min(max(left + 8 * (threadIdx.x & 31), 0ll), 256ll));
        if (kAhead) {
            if (kPost && a.post_w) load_vector_pairs(a.post_w, col[c], exist[c], vectors, 1.0f, post_w[c]);
            if (kPre && a.pre_w) load_vector_pairs(a.pre_w, col[c], exist[c], vectors, 1.0f, pre_w[c]);
        }
    }
    struct Row {
        Eight<kType> x[kRuns], z[kRuns], g[kRuns];
    };
    constexpr int kSize = kType == kF32 ? 4 : 2;
    const long long run = 8ll * blockDim.x;              // columns between a thread's runs
    const long long step = static_cast<long long>(gridDim.x) * blockDim.y;
    const long long first = static_cast<long long>(blockIdx.x) * blockDim.y + threadIdx.y;
    // (addresses of the next row to read and of this row's outputs go on by a step's bytes)
    const char* z_at = static_cast<const char*>(a.Z) + (first * a.ldz + col[0]) * kSize;
    const char* x_at = static_cast<const char*>(a.X) + (first * a.ldx + col[0]) * kSize;
    char* y_at = static_cast<char*>(a.Y) + (first * a.ldy + col[0]) * kSize;
    char* h_at = static_cast<char*>(a.H) + (first * a.ldh + col[0]) * kSize;
    const long long z_step = step * a.ldz * kSize, x_step = step * a.ldx * kSize, y_step = step * a.ldy * kSize, h_step = step * a.ldh * kSize;
    const int gate_kind = a.gate_rows >= a.M ? 0 : (a.gate_rows == 1 ? 1 : 2);       // one row for all, one each, some share one
    const auto load = [&](Row& r, long long row) {
        const bool here = row < a.M;
        uint32_t gate_row = gate_kind == 0 || !here ? 0u : static_cast<uint32_t>(row);
        if (gate_kind == 2) gate_row /= static_cast<uint32_t>(a.gate_rows);
        const char* const g_at = static_cast<const char*>(a.gate) + (gate_row * a.ldgate + col[0]) * kSize;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            const int count = here ? exist[c] : 0;
            const int limit = here ? warp_exist[c] : 0;
            if (a.Z) load_run<kWide>(r.z[c], z_at + c * run * kSize, count, limit);
            else r.z[c].clear();
            if (a.X) load_run<kWide>(r.x[c], x_at + c * run * kSize, count, limit);
            else r.x[c].clear();
            if (a.gate) load_run<kWide>(r.g[c], g_at + c * run * kSize, count, limit);
        }
        z_at += z_step;
        x_at += x_step;
    };
    Row cur;
    load(cur, first);
    for (long long row = first; row - threadIdx.y < a.M; row += step, y_at += y_step, h_at += h_step) {
        const bool here = row < a.M;
        int count[kRuns];
        uint64_t v[kRuns][4];
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            count[c] = here ? exist[c] : 0;
            run_pairs<kWide>(cur.z[c], buf, v[c]);
        }
        Row next;
        if (kAhead) load(next, row + step);
        float2 post = make_float2(0.0f, 0.0f), pre = post;
        if (kPost && a.post != kNormNone) {
            post = normalize<kRuns>(a.post, v, count, inv_n, a.eps, ex, slot);
            affine<kRuns>(v, post_w, kAhead, a.post_w, a.post_b, col, exist, vectors);
        }
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            uint64_t t[4];
            if (a.gate) {
                run_pairs<kWide>(cur.g[c], buf, t);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[c][j] = mul_f2(v[c][j], t[j]);
            }
            if (drop.bar) drop.apply(drop.draw(row, col[c]), v[c]);
            if (a.X) {
                run_pairs<kWide>(cur.x[c], buf, t);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[c][j] = fma_f2(pack_f2(a.x_scale, a.x_scale), t[j], v[c][j]);
            }
            if (a.Y)
                store_run<kWide, kType>(v[c], y_at + c * run * kSize, count[c], here ? warp_exist[c] : 0, buf);
        }
        if (kPre && a.pre != kNormNone) {
            pre = normalize<kRuns>(a.pre, v, count, inv_n, a.eps, ex, slot);
            affine<kRuns>(v, pre_w, kAhead, a.pre_w, a.pre_b, col, exist, vectors);
            if (a.H) {
#pragma unroll
                for (int c = 0; c < kRuns; ++c) {
                    store_run<kWide, kType>(v[c], h_at + c * run * kSize, count[c], here ? warp_exist[c] : 0, buf);
                }
            }
            if (a.codes != kCodesNone) {
                float top[kRuns], most = 0.0f;
#pragma unroll
                for (int c = 0; c < kRuns; ++c) {
                    if (!kWide) clear_behind(v[c], count[c]);
                    top[c] = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float lo, hi;
                        unpack_f2(v[c][j], lo, hi);
                        top[c] = max_magnitude(max_magnitude(top[c], lo), hi);
                    }
                    most = max_magnitude(most, top[c]);
                }
                if (a.codes == kCodesS8) {
                    const float top_f = __uint_as_float(row_max(magnitude_bits(most), ex, slot));
                    // (the rule of mipgemm_quantize_rows)
                    float scale = 0.0f, mult = 0.0f;
                    if (!(top_f <= 3.402823466e38f)) {
                        scale = __int_as_float(0x7FFFFFFF);
                    } else if (top_f >= 0x1p-119f) {
                        scale = __fdiv_rn(top_f, 127.0f);
                        mult = __fdiv_rn(127.0f, top_f);
                    }
                    if (here && threadIdx.x == 0) a.q_scale[row] = scale;
#pragma unroll
                    for (int c = 0; c < kRuns; ++c) {
                        float h[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) unpack_f2(mul_f2(v[c][j], pack_f2(mult, mult)), h[2 * j], h[2 * j + 1]);
                        uint32_t q[2] = {0u, 0u};
                        if (mult != 0.0f) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) q[j / 4] |= (static_cast<uint32_t>(__float2int_rn(h[j])) & 0xFFu) << (8 * (j & 3));
                        }
                        store_codes8(a.Q + row * a.ldq + col[c], make_uint2(q[0], q[1]), count[c], wide);
                    }
                } else {
                    // a block of 128 columns is what 16 neighbouring lanes hold
#pragma unroll
                    for (int c = 0; c < kRuns; ++c) {
#pragma unroll
                        for (int o = 8; o > 0; o >>= 1) top[c] = max_magnitude(top[c], __shfl_xor_sync(~0u, top[c], o));
                    }
                    const auto put = [&](auto format) {
                        constexpr int kFormat = decltype(format)::value;
#pragma unroll
                        for (int c = 0; c < kRuns; ++c) {
                            const F8Scale s = f8_scale<kFormat>(top[c]);
                            if ((threadIdx.x & 15) == 0 && count[c] > 0) a.q_scale[(col[c] >> 7) * a.ldqs + row] = s.scale;
                            uint32_t q[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float lo, hi;
                                unpack_f2(mul_f2(v[c][j], pack_f2(s.mult, s.mult)), lo, hi);
                                q[j] = f8_pair<kFormat>(lo, hi);
                            }
                            // (a multiplier of 0 stands for "codes 0": an infinity times 0 would be NaN)
                            const uint2 w = s.mult == 0.0f ? make_uint2(0u, 0u) : make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
                            store_codes8(a.Q + row * a.ldq + col[c], w, count[c], wide);
                        }
                    };
                    if (a.codes == kCodesE4M3) put(std::integral_constant<int, kE4M3>{});
                    else put(std::integral_constant<int, kE5M2>{});
                }
            }
        }
        if (a.stats && here && threadIdx.x == 0 && blockIdx.y == 0) {
            float* s = a.stats + 4 * row;
            s[0] = post.x; s[1] = post.y; s[2] = pre.x; s[3] = pre.y;
        }
        if (kAhead) cur = next;
        else if (row - threadIdx.y + step < a.M) load(cur, row + step);
    }
}

struct StepShape {
    int runs, threads, rows, blocks;     // blocks: 0, one for each `rows` rows; else they go on from row to row
    int parts;                           // of a row, each a block's
    bool apart;                          // without norms
};
// 16 columns a thread where there are rows enough to go on with; else eight, and more threads on a row.  Without norms nothing
// holds a row together: blocks take 4096 columns of it.
StepShape step_shape(const StepArgs& a, int sm_count) {
    StepShape s;
    const long long M = a.M;
    const bool apart = s.apart = a.post == kNormNone && a.pre == kNormNone;
    s.parts = apart ? static_cast<int>((a.N + 4095) / 4096) : 1;
    const long long N = apart ? std::min<long long>(a.N, 4096) : a.N;
    const bool many = M * s.parts >= 4ll * sm_count && N <= 8192;
    s.runs = many || apart ? 2 : (N <= 4096 ? 1 : (N <= 8192 ? 2 : 4));
    const long long per = 8ll * s.runs;
    s.threads = static_cast<int>(((N + per - 1) / per + 31) / 32 * 32);
    s.rows = std::max(1, std::min(kMaxBlockRows, (many || apart ? 256 : 128) / s.threads));
    s.blocks = many ? std::max(1, sm_count * (apart ? 8 : (s.threads > 256 ? 1 : 2)) / s.parts) : 0;
    return s;
}

template <int kType, bool kWide>
cudaError_t step_t(const StepArgs& a, const StepShape& s, const cudaLaunchConfig_t& cfg) {
    if (s.apart) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 2, 256, false, kWide, false, false>, a);
    if (s.blocks) {
        const bool post = a.post != kNormNone, pre = a.pre != kNormNone;
        const auto many = [&](auto has_post, auto has_pre) {
            constexpr bool kPost = decltype(has_post)::value, kPre = decltype(has_pre)::value;
            if (s.threads <= 256) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 2, 256, true, kWide, kPost, kPre>, a);
            return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 2, 512, true, kWide, kPost, kPre>, a);
        };
        if (post && pre) return many(std::true_type{}, std::true_type{});
        return post ? many(std::true_type{}, std::false_type{}) : many(std::false_type{}, std::true_type{});
    }
    if (s.runs == 1) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 1, 512, false, kWide, true, true>, a);
    if (s.runs == 2) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 2, 512, false, kWide, true, true>, a);
    if (s.threads <= 512) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 4, 512, false, kWide, true, true>, a);
    return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 4, 1024, false, kWide, true, true>, a);
}
template <int kType>
cudaError_t step_wide(const StepArgs& a, const StepShape& s, const cudaLaunchConfig_t& cfg) {
    return a.wide ? step_t<kType, true>(a, s, cfg) : step_t<kType, false>(a, s, cfg);
}

}  // namespace

void step_mask(StepMask& m, unsigned long long seed, const unsigned long long* counter) {
    philox_keys(seed, m.keys);
    m.counter = counter;
}

cudaError_t launch_norm_step(int type, const StepArgs& a, int sm_count, cudaStream_t stream) {
    const StepShape s = step_shape(a, sm_count);
    cudaLaunchConfig_t cfg = {};
    const long long blocks = (a.M + s.rows - 1) / s.rows;
    cfg.gridDim = dim3(static_cast<unsigned>(s.blocks ? std::min<long long>(s.blocks, blocks) : blocks), static_cast<unsigned>(s.parts));
    cfg.blockDim = dim3(static_cast<unsigned>(s.threads), static_cast<unsigned>(s.rows));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = cfg.gridDim.x * cfg.gridDim.y <= 128 ? 1 : 0;                   // (launched early only where the blocks are few, like the row kernels)
    if (type == kF32) return step_wide<kF32>(a, s, cfg);
    return type == kF16 ? step_wide<kF16>(a, s, cfg) : step_wide<kBF16>(a, s, cfg);
}

}  // namespace mip
