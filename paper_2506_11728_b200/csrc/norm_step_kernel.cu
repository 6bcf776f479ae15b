// The step between two blocks of a transformer layer, forward:
//     v = dropout(gate * norm_post(z)),  y = s x + v,  h = norm_pre(y),  h as values and/or as 8-bit codes,
// every part optional.  Two norms, a gate, a mask, the residual sum and the codes in one pass: x and z are read once, y and h
// (or h's codes) written once, and the mask exists nowhere but in registers.
//
// A row stays in the registers of its threads, eight neighbouring columns each and up to four such runs (rows of up to 32768
// columns).  Means come first, then the squares of what is left, so that a large mean takes no digits from the variance.
// The dropout mask is a function of (seed, counter, row, column): one draw of a counter-based generator for eight columns.
//
// What bounds it: the bytes of x, z, y and h.
#include "ptx.cuh"
#include "step_math.cuh"

namespace mip {

namespace {

// Sum over a row's threads; all of them get it.  `slot`: which of the exchange buffers, another one for each use.
__device__ __forceinline__ float row_sum(float v, float (*part)[kMaxBlockRows][kMaxRowWarps], int slot) {
    v = warp_sum(v);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) part[slot][threadIdx.y][threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < warps ? part[slot][threadIdx.y][lane] : 0.0f);
}
__device__ __forceinline__ uint32_t row_max(uint32_t v, float (*part)[kMaxBlockRows][kMaxRowWarps], int slot) {
    v = __reduce_max_sync(~0u, v);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) part[slot][threadIdx.y][threadIdx.x >> 5] = __uint_as_float(v);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return __reduce_max_sync(~0u, lane < warps ? __float_as_uint(part[slot][threadIdx.y][lane]) : 0u);
}

// v becomes w (v - mean) / sqrt(var + eps) + b; returns (mean, 1 / sqrt(var + eps)).
template <int kRuns>
__device__ __forceinline__ float2 normalize(int kind, float (&v)[kRuns][8], const int (&count)[kRuns], const float* w, const float* b, bool wide,
                                            const long long (&col)[kRuns], long long N, float eps, float (*part)[kMaxBlockRows][kMaxRowWarps], int slot) {
    float mean = 0.0f;
    if (kind == kNormLayer) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < kRuns; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[c][j];                  // (columns that do not exist hold 0)
        mean = __fdiv_rn(row_sum(s, part, slot), static_cast<float>(N));
    }
    float q = 0.0f;
#pragma unroll
    for (int c = 0; c < kRuns; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[c][j] = j < count[c] ? v[c][j] - mean : 0.0f;
            q = fmaf(v[c][j], v[c][j], q);
        }
    const float rstd = __frsqrt_rn(__fadd_rn(__fdiv_rn(row_sum(q, part, slot + 1), static_cast<float>(N)), eps));
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        float wv[8], bv[8];
        load_vector8(w, col[c], count[c], wide, 1.0f, wv);
        load_vector8(b, col[c], count[c], wide, 0.0f, bv);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = fmaf(v[c][j] * rstd, wv[j], bv[j]);
    }
    return make_float2(mean, rstd);
}

template <int kFormat>
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float mult) {
    return make_uint2(f8_codes4<kFormat>(v[0], v[1], v[2], v[3], mult), f8_codes4<kFormat>(v[4], v[5], v[6], v[7], mult));
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

template <int kType, int kRuns, int kThreads>
__global__ void __launch_bounds__(kThreads)
mip_norm_step_kernel(const StepArgs a) {
    __shared__ float part[5][kMaxBlockRows][kMaxRowWarps];
    pdl_wait();
    pdl_launch_dependents();
    const long long row = static_cast<long long>(blockIdx.x) * blockDim.y + threadIdx.y;
    const bool here = row < a.M;
    const bool wide = a.wide;
    const bool gated = a.gate && here;
    const Dropout drop = dropout_of(a.bar, a.drop_scale, a.seed, a.counter, a.N);
    long long col[kRuns];
    int count[kRuns];
    Eight<kType> x[kRuns], z[kRuns], g[kRuns];
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        col[c] = 8ll * (static_cast<long long>(c) * blockDim.x + threadIdx.x);
        const long long left = here ? a.N - col[c] : 0;
        count[c] = left <= 0 ? 0 : (left < 8 ? static_cast<int>(left) : 8);
        if (a.Z) z[c].load(a.Z, row * a.ldz + col[c], count[c], wide);
        else z[c].clear();
        if (a.X) x[c].load(a.X, row * a.ldx + col[c], count[c], wide);
        else x[c].clear();
        if (gated) g[c].load(a.gate, static_cast<uint32_t>(row) / static_cast<uint32_t>(a.gate_rows) * a.ldgate + col[c], count[c], wide);
    }
    float v[kRuns][8];
#pragma unroll
    for (int c = 0; c < kRuns; ++c) z[c].values(v[c]);
    float2 post = make_float2(0.0f, 0.0f), pre = post;
    if (a.post != kNormNone) post = normalize<kRuns>(a.post, v, count, a.post_w, a.post_b, wide, col, a.N, a.eps, part, 0);
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
        if (gated) {
            float gv[8];
            g[c].values(gv);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= gv[j];
        }
        if (drop.bar) drop.apply(drop.draw(row, col[c]), v[c]);
        float xv[8];
        x[c].values(xv);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = fmaf(a.x_scale, xv[j], v[c][j]);
        if (a.Y) {
            Eight<kType> y;
            y.set(v[c]);
            y.store(a.Y, row * a.ldy + col[c], count[c], wide);
        }
    }
    if (a.pre != kNormNone) {
        pre = normalize<kRuns>(a.pre, v, count, a.pre_w, a.pre_b, wide, col, a.N, a.eps, part, 2);
        if (a.H) {
#pragma unroll
            for (int c = 0; c < kRuns; ++c) {
                Eight<kType> h;
                h.set(v[c]);
                h.store(a.H, row * a.ldh + col[c], count[c], wide);
            }
        }
        if (a.codes == kCodesS8) {
            uint32_t top = 0u;
#pragma unroll
            for (int c = 0; c < kRuns; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) top = max(top, j < count[c] ? magnitude_bits(v[c][j]) : 0u);
            const float top_f = __uint_as_float(row_max(top, part, 4));
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
                uint32_t q[2] = {0u, 0u};
                if (mult != 0.0f) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[j / 4] |= (static_cast<uint32_t>(__float2int_rn(__fmul_rn(v[c][j], mult))) & 0xFFu) << (8 * (j & 3));
                }
                store_codes8(a.Q + row * a.ldq + col[c], make_uint2(q[0], q[1]), count[c], wide);
            }
        } else if (a.codes != kCodesNone) {
            // a block of 128 columns is what 16 neighbouring lanes hold
#pragma unroll
            for (int c = 0; c < kRuns; ++c) {
                uint32_t top = 0u;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = max(top, j < count[c] ? magnitude_bits(v[c][j]) : 0u);
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
                const bool e4m3 = a.codes == kCodesE4M3;
                const F8Scale s = e4m3 ? f8_scale<kE4M3>(__uint_as_float(top)) : f8_scale<kE5M2>(__uint_as_float(top));
                if ((threadIdx.x & 15) == 0 && count[c] > 0) a.q_scale[(col[c] >> 7) * a.ldqs + row] = s.scale;
                store_codes8(a.Q + row * a.ldq + col[c], e4m3 ? codes8<kE4M3>(v[c], s.mult) : codes8<kE5M2>(v[c], s.mult), count[c], wide);
            }
        }
    }
    if (a.stats && here && threadIdx.x == 0) {
        float* s = a.stats + 4 * row;
        s[0] = post.x; s[1] = post.y; s[2] = pre.x; s[3] = pre.y;
    }
}

template <int kType>
cudaError_t step_t(const StepArgs& a, int runs, const cudaLaunchConfig_t& cfg) {
    if (runs == 1) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 1, 512>, a);
    if (runs == 2) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 2, 512>, a);
    if (cfg.blockDim.x <= 512) return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 4, 512>, a);
    return cudaLaunchKernelEx(&cfg, mip_norm_step_kernel<kType, 4, 1024>, a);
}

}  // namespace

cudaError_t launch_norm_step(int type, const StepArgs& a, cudaStream_t stream) {
    const int runs = a.N <= 4096 ? 1 : (a.N <= 8192 ? 2 : 4);
    const long long per = 8ll * runs;
    const int threads = static_cast<int>(((a.N + per - 1) / per + 31) / 32 * 32);
    const int rows = threads >= 128 ? 1 : 128 / threads;           // (at most kMaxBlockRows)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((a.M + rows - 1) / rows));
    cfg.blockDim = dim3(static_cast<unsigned>(threads), static_cast<unsigned>(rows));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = cfg.gridDim.x <= 128 ? 1 : 0;                   // (launched early only where the blocks are few, like the row kernels)
    if (type == kF32) return step_t<kF32>(a, runs, cfg);
    return type == kF16 ? step_t<kF16>(a, runs, cfg) : step_t<kBF16>(a, runs, cfg);
}

}  // namespace mip
