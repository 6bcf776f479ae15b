// Matrices to 8-bit floating point with a float32 scale for each block of 128 elements along the rows, along the columns
// or of 128 x 128, and back.
//
// A CTA takes a tile of 128 x 128 and reads it once: it stays in registers (64 elements per thread) between the blocks'
// largest magnitudes and the codes, so that codes along both axes cost one reading.  A row's block lies in neighbouring
// lanes (shuffles), a column's in all warps (a 4 KB exchange in shared memory), a square in the whole CTA.  Magnitudes are
// compared as bit patterns, where infinities and NaNs come out on top.
//
// What bounds it: the bytes (16384 x 4096 bf16: along the rows 34 us, 5.8 TB/s, squares 32, back 40 to 43), and for codes along both
// axes the conversions beside them (57 us where their bytes take 41; along the columns alone 41).
#include "float8_math.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace mip {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPerThread = kF8Block * kF8Block / kThreads;       // 64

// Where a thread's elements lie in the tile: kRuns runs of kLen consecutive columns.
//   wide: 4 runs of 16 columns, 32 rows apart (16- or 32-byte accesses, eight lanes a row)
//   else: 64 single elements, 32 columns or 8 rows apart (a warp a row, any alignment)
template <bool kWide>
struct Place {
    static constexpr int kRuns = kWide ? 4 : 16;                 // rows per thread
    static constexpr int kLen = kPerThread / kRuns;              // columns per thread and row
    static __device__ __forceinline__ int row(int i) { return kWide ? static_cast<int>(threadIdx.x >> 3) + 32 * i : static_cast<int>(threadIdx.x >> 5) + kWarps * i; }
    static __device__ __forceinline__ int col(int j) { return kWide ? static_cast<int>(threadIdx.x & 7) * 16 + j : static_cast<int>(threadIdx.x & 31) + 32 * j; }
};

// A thread's elements of a tile as they came (unpacked where they are used: 16-bit elements take half the registers);
// what lies outside the matrix is 0.
template <int kType, bool kWide>
struct Tile {
    using P = Place<kWide>;
    Eight<kType> e[P::kRuns][kWide ? 2 : 1];             // (single elements: 4 of the 8 places)
    __device__ __forceinline__ void load(const void* X, long long ldx, long long r0, long long c0, long long M, long long N) {
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i) {
            const long long r = r0 + P::row(i);
            if constexpr (kWide) {
                const long long c = c0 + P::col(0);
#pragma unroll
                for (int h = 0; h < 2; ++h) e[i][h].load(X, r * ldx + c + 8 * h, r < M && c + 8 * h < N ? 8 : 0);
            } else {
                float v[8] = {};
#pragma unroll
                for (int j = 0; j < P::kLen; ++j) {
                    const long long c = c0 + P::col(j);
                    if (r < M && c < N) v[j] = load_one<kType>(X, r * ldx + c);
                }
                e[i][0].set(v);                          // (exact: the elements are of the type)
            }
        }
    }
    __device__ __forceinline__ void values(int i, float (&v)[P::kLen]) const {
        float x[8];
        e[i][0].values(x);
#pragma unroll
        for (int j = 0; j < (kWide ? 8 : 4); ++j) v[j] = x[j];
        if constexpr (kWide) {
            e[i][1].values(x);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 + j] = x[j];
        }
    }
};
// Magnitudes on the elements' own bits, two of 16 bits at a time (they order like the magnitudes, infinities and NaNs on top).
template <int kType>
__device__ __forceinline__ uint32_t word_max(uint32_t top, uint32_t w) {
    return kType == kF32 ? max(top, w & 0x7FFFFFFFu) : __vmaxu2(top, w & 0x7FFF7FFFu);
}
template <int kType>
__device__ __forceinline__ float word_top(uint32_t top) {            // of the two halves
    if (kType == kF32) return __uint_as_float(top);
    const uint32_t m = max(top & 0xFFFFu, top >> 16);
    return kType == kF16 ? __half2float(__ushort_as_half(static_cast<uint16_t>(m))) : __uint_as_float(m << 16);
}

// kForm: bit 0 blocks along the rows, bit 1 along the columns; 4: squares.
struct CodesArgs {
    long long M, N;
    const void* X; long long ldx;
    uint8_t* Q[2]; long long ldq[2];         // along the rows (or squares), along the columns
    float* scale[2]; long long lds[2];
};

template <int kType, int kFormat, int kForm, bool kWide>
__global__ void __launch_bounds__(kThreads, kType == kF32 ? 2 : (kForm & 2 ? 3 : 4))
mip_f8_quantize_kernel(const CodesArgs a) {
    using P = Place<kWide>;
    constexpr bool kRows = kForm & 1, kCols = kForm & 2, kSquare = kForm & 4;
    __shared__ uint32_t part[kCols ? kWarps : 1][kCols ? kF8Block : kWarps];
    pdl_wait();
    pdl_launch_dependents();
    const long long r0 = static_cast<long long>(blockIdx.y) * kF8Block, c0 = static_cast<long long>(blockIdx.x) * kF8Block;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Tile<kType, kWide> t;
    t.load(a.X, a.ldx, r0, c0, a.M, a.N);

    // Codes of run i, one multiplier for each column.
    const auto put = [&](int side, int i, const auto& mult_of) {
        const long long r = r0 + P::row(i);
        if (r >= a.M) return;
        uint8_t* dst = a.Q[side] + r * a.ldq[side] + c0;
        float v[P::kLen];
        t.values(i, v);
        if constexpr (kWide) {
            const int c = P::col(0);
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (side == 0) {
                    q[j] = f8_codes4<kFormat>(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3], mult_of(0));
                    continue;
                }
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    // (a multiplier of 0 stands for "codes 0": an infinity times 0 would be NaN)
                    const float m0 = mult_of(4 * j + e), m1 = mult_of(4 * j + e + 1);
                    w[e / 2] = f8_pair<kFormat>(m0 == 0.0f ? 0.0f : __fmul_rn(v[4 * j + e], m0), m1 == 0.0f ? 0.0f : __fmul_rn(v[4 * j + e + 1], m1));
                }
                q[j] = w[0] | (w[1] << 16);
            }
            if (c0 + c + 16 <= a.N) *reinterpret_cast<uint4*>(dst + c) = make_uint4(q[0], q[1], q[2], q[3]);
            else if (c0 + c < a.N) *reinterpret_cast<uint2*>(dst + c) = make_uint2(q[0], q[1]);     // (N is a multiple of 8)
        } else {
#pragma unroll
            for (int j = 0; j < P::kLen; ++j) {
                const float m = mult_of(j);
                if (c0 + P::col(j) < a.N)
                    dst[P::col(j)] = m == 0.0f ? uint8_t(0) : static_cast<uint8_t>(f8_pair<kFormat>(__fmul_rn(v[j], m), 0.0f));
            }
        }
    };
    constexpr int kWords = kType == kF32 ? 8 : 4;        // of eight elements
    constexpr int kUsed = kWide ? kWords : kWords / 2;

    if constexpr (kRows) {
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i) {
            uint32_t top = 0u;
#pragma unroll
            for (int h = 0; h < (kWide ? 2 : 1); ++h)
#pragma unroll
                for (int j = 0; j < kUsed; ++j) top = word_max<kType>(top, t.e[i][h].w[j]);
            if constexpr (kWide) {
#pragma unroll
                for (int o = 4; o > 0; o >>= 1) top = word_max<kType>(top, __shfl_xor_sync(~0u, top, o));
            } else {
                if (kType != kF32) top = max(top & 0xFFFFu, top >> 16);
                top = __reduce_max_sync(~0u, top);
            }
            const F8Scale s = f8_scale<kFormat>(word_top<kType>(top));
            const long long r = r0 + P::row(i);
            if (r < a.M && (threadIdx.x & (kWide ? 7 : 31)) == 0) a.scale[0][static_cast<long long>(blockIdx.x) * a.lds[0] + r] = s.scale;
            put(0, i, [&](int) { return s.mult; });
        }
    }
    if constexpr (kCols) {
        // largest magnitude of each column: over the thread's rows, over the warp's, over the warps'
#pragma unroll
        for (int h = 0; h < (kWide ? 2 : 1); ++h) {
#pragma unroll
            for (int j = 0; j < kUsed; ++j) {
                uint32_t top = 0u;
#pragma unroll
                for (int i = 0; i < P::kRuns; ++i) top = word_max<kType>(top, t.e[i][h].w[j]);
                if constexpr (kWide) {
                    top = word_max<kType>(top, __shfl_xor_sync(~0u, top, 8));
                    top = word_max<kType>(top, __shfl_xor_sync(~0u, top, 16));
                }
                if (!kWide || lane < 8) {
                    if constexpr (kType == kF32) {
                        part[warp][P::col(8 * h + j)] = top;
                    } else {
                        part[warp][P::col(8 * h + 2 * j)] = top & 0xFFFFu;
                        part[warp][P::col(8 * h + 2 * j + 1)] = top >> 16;
                    }
                }
            }
        }
        __syncthreads();
        float* mult = reinterpret_cast<float*>(part[0]);
        if (threadIdx.x < kF8Block) {
            uint32_t m = 0u;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = max(m, part[w][threadIdx.x]);
            const F8Scale s = f8_scale<kFormat>(word_top<kType>(m));
            mult[threadIdx.x] = s.mult;
            if (c0 + threadIdx.x < a.N) a.scale[1][static_cast<long long>(blockIdx.y) * a.lds[1] + c0 + threadIdx.x] = s.scale;
        }
        __syncthreads();
        float m[P::kLen];
#pragma unroll
        for (int j = 0; j < P::kLen; ++j) m[j] = mult[P::col(j)];
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i) put(1, i, [&](int j) { return m[j]; });
    }
    if constexpr (kSquare) {
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i)
#pragma unroll
            for (int h = 0; h < (kWide ? 2 : 1); ++h)
#pragma unroll
                for (int j = 0; j < kUsed; ++j) top = word_max<kType>(top, t.e[i][h].w[j]);
        if (kType != kF32) top = max(top & 0xFFFFu, top >> 16);
        top = __reduce_max_sync(~0u, top);
        if (lane == 0) part[0][warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = max(top, part[0][w]);
        const F8Scale s = f8_scale<kFormat>(word_top<kType>(top));
        if (threadIdx.x == 0) a.scale[0][static_cast<long long>(blockIdx.y) * a.lds[0] + blockIdx.x] = s.scale;
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i) put(0, i, [&](int) { return s.mult; });
    }
}

template <int kType, int kFormat, bool kWide>
__global__ void __launch_bounds__(kThreads)
mip_f8_dequantize_kernel(int blocks, long long M, long long N, const uint8_t* Q, long long ldq, const float* scale, long long lds, void* X, long long ldx) {
    using P = Place<kWide>;
    pdl_wait();
    pdl_launch_dependents();
    const long long r0 = static_cast<long long>(blockIdx.y) * kF8Block, c0 = static_cast<long long>(blockIdx.x) * kF8Block;
    const long long rb = blockIdx.y, cb = blockIdx.x;
    uint32_t q[P::kRuns][kWide ? 4 : P::kLen];
#pragma unroll
    for (int i = 0; i < P::kRuns; ++i) {
        const long long r = r0 + P::row(i);
        const uint8_t* src = Q + r * ldq + c0;
        if constexpr (kWide) {
            const int c = P::col(0);
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (r < M && c0 + c + 16 <= N) {
                w = ld_once_v4(src + c);
            } else if (r < M && c0 + c < N) {
                const uint2 h = *reinterpret_cast<const uint2*>(src + c);
                w.x = h.x;
                w.y = h.y;
            }
            q[i][0] = w.x; q[i][1] = w.y; q[i][2] = w.z; q[i][3] = w.w;
        } else {
#pragma unroll
            for (int j = 0; j < P::kLen; ++j) q[i][j] = r < M && c0 + P::col(j) < N ? src[P::col(j)] : 0u;
        }
    }
    // (all scales are asked for at once, beside the codes)
    float by_col[P::kLen], by_row[P::kRuns];
    if (blocks == kBlocksRows) {
#pragma unroll
        for (int i = 0; i < P::kRuns; ++i) by_row[i] = r0 + P::row(i) < M ? __ldg(scale + cb * lds + r0 + P::row(i)) : 0.0f;
    } else if (blocks == kBlocksColumns) {
#pragma unroll
        for (int j = 0; j < P::kLen; ++j) by_col[j] = c0 + P::col(j) < N ? __ldg(scale + rb * lds + c0 + P::col(j)) : 0.0f;
    } else if (blocks == kBlocksSquares) {
        const float s = __ldg(scale + rb * lds + cb);
#pragma unroll
        for (int j = 0; j < P::kLen; ++j) by_col[j] = s;
    }
#pragma unroll
    for (int i = 0; i < P::kRuns; ++i) {
        const long long r = r0 + P::row(i);
        if (r >= M) continue;
        if (blocks == kBlocksRows) {
#pragma unroll
            for (int j = 0; j < P::kLen; ++j) by_col[j] = by_row[i];
        }
        if constexpr (kWide) {
            const long long c = c0 + P::col(0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float2 x = f8_values<kFormat>(q[i][2 * h + j / 4] >> (16 * (j / 2 & 1)));
                    v[j] = __fmul_rn(x.x, by_col[8 * h + j]);
                    v[j + 1] = __fmul_rn(x.y, by_col[8 * h + j + 1]);
                }
                Eight<kType> e;
                e.set(v);
                e.store(X, r * ldx + c + 8 * h, c + 8 * h < N ? 8 : 0, true);
            }
        } else {
#pragma unroll
            for (int j = 0; j < P::kLen; ++j)
                if (c0 + P::col(j) < N) store_one<kType>(X, r * ldx + c0 + P::col(j), __fmul_rn(f8_values<kFormat>(q[i][j]).x, by_col[j]));
        }
    }
}

bool aligned_rows(const void* p, long long pitch_bytes, int bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && pitch_bytes % bytes == 0;
}

// (launched early only where the blocks are few, like the row kernels)
template <typename... Formal, typename... Actual>
cudaError_t launch(void (*kernel)(Formal...), dim3 grid, cudaStream_t stream, Actual... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = static_cast<long long>(grid.x) * grid.y <= 128 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Formal>(args)...);
}

// The grid's second dimension holds 65535 blocks: more rows go in several launches.
constexpr long long kRowsPerLaunch = 65535LL * kF8Block;

template <int kType, int kFormat, int kForm>
cudaError_t quantize_t(const CodesArgs& a, bool wide, dim3 grid, cudaStream_t stream) {
    return wide ? launch(mip_f8_quantize_kernel<kType, kFormat, kForm, true>, grid, stream, a)
                : launch(mip_f8_quantize_kernel<kType, kFormat, kForm, false>, grid, stream, a);
}
template <int kType, int kFormat>
cudaError_t quantize_form(const CodesArgs& a, int form, bool wide, dim3 grid, cudaStream_t stream) {
    if (form == 1) return quantize_t<kType, kFormat, 1>(a, wide, grid, stream);
    if (form == 2) return quantize_t<kType, kFormat, 2>(a, wide, grid, stream);
    if (form == 3) return quantize_t<kType, kFormat, 3>(a, wide, grid, stream);
    return quantize_t<kType, kFormat, 4>(a, wide, grid, stream);
}

}  // namespace

// form: bit 0 blocks along the rows (side 0), bit 1 along the columns (side 1); 4: squares (side 0)
cudaError_t launch_f8_quantize(int type, int format, int form, long long M, long long N, const void* X, long long ldx, const F8Codes (&out)[2],
                               cudaStream_t stream, int* launches) {
    const int size = type == kF32 ? 4 : 2;
    bool wide = N % 8 == 0 && aligned_rows(X, ldx * size, 16);
    for (int side = 0; side < 2; ++side)
        if (out[side].Q) wide = wide && aligned_rows(out[side].Q, out[side].ldq, 16);
    for (long long row = 0; row < M; row += kRowsPerLaunch) {
        const long long rb = row / kF8Block;
        CodesArgs a;
        a.M = M - row < kRowsPerLaunch ? M - row : kRowsPerLaunch;
        a.N = N;
        a.X = static_cast<const char*>(X) + row * ldx * size;
        a.ldx = ldx;
        for (int side = 0; side < 2; ++side) {
            a.Q[side] = out[side].Q ? static_cast<uint8_t*>(out[side].Q) + row * out[side].ldq : nullptr;
            a.ldq[side] = out[side].ldq;
            a.scale[side] = out[side].scale ? out[side].scale + (side == 0 && form != 4 ? row : rb * out[side].lds) : nullptr;
            a.lds[side] = out[side].lds;
        }
        const dim3 grid(static_cast<unsigned>((N + kF8Block - 1) / kF8Block), static_cast<unsigned>((a.M + kF8Block - 1) / kF8Block));
        cudaError_t e;
        if (format == kE4M3)
            e = type == kF32 ? quantize_form<kF32, kE4M3>(a, form, wide, grid, stream)
                             : (type == kF16 ? quantize_form<kF16, kE4M3>(a, form, wide, grid, stream) : quantize_form<kBF16, kE4M3>(a, form, wide, grid, stream));
        else
            e = type == kF32 ? quantize_form<kF32, kE5M2>(a, form, wide, grid, stream)
                             : (type == kF16 ? quantize_form<kF16, kE5M2>(a, form, wide, grid, stream) : quantize_form<kBF16, kE5M2>(a, form, wide, grid, stream));
        ++*launches;
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_f8_dequantize(int type, int format, int blocks, long long M, long long N, const F8Codes& in, void* X, long long ldx,
                                 cudaStream_t stream, int* launches) {
    const int size = type == kF32 ? 4 : 2;
    const bool wide = N % 8 == 0 && aligned_rows(X, ldx * size, 16) && aligned_rows(in.Q, in.ldq, 16);
    for (long long row = 0; row < M; row += kRowsPerLaunch) {
        const long long m = M - row < kRowsPerLaunch ? M - row : kRowsPerLaunch;
        const uint8_t* q = static_cast<const uint8_t*>(in.Q) + row * in.ldq;
        const float* scale = in.scale + (blocks == kBlocksRows ? row : row / kF8Block * in.lds);
        void* x = static_cast<char*>(X) + row * ldx * size;
        const dim3 grid(static_cast<unsigned>((N + kF8Block - 1) / kF8Block), static_cast<unsigned>((m + kF8Block - 1) / kF8Block));
        cudaError_t e;
#define MIP_DEQUANTIZE(T, F)                                                                                                  \
    (wide ? launch(mip_f8_dequantize_kernel<T, F, true>, grid, stream, blocks, m, N, q, in.ldq, scale, in.lds, x, ldx)        \
          : launch(mip_f8_dequantize_kernel<T, F, false>, grid, stream, blocks, m, N, q, in.ldq, scale, in.lds, x, ldx))
        if (format == kE4M3) e = type == kF32 ? MIP_DEQUANTIZE(kF32, kE4M3) : (type == kF16 ? MIP_DEQUANTIZE(kF16, kE4M3) : MIP_DEQUANTIZE(kBF16, kE4M3));
        else e = type == kF32 ? MIP_DEQUANTIZE(kF32, kE5M2) : (type == kF16 ? MIP_DEQUANTIZE(kF16, kE5M2) : MIP_DEQUANTIZE(kBF16, kE5M2));
#undef MIP_DEQUANTIZE
        ++*launches;
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace mip
