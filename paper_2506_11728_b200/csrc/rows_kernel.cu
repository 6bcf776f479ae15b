// Rows of activations to 8-bit codes with one scale each, and back.  Both are bound by the bytes they move (16-bit
// types: 2 in, 1 out per element, or the reverse): 16384 x 4096 bf16 there and back 64 to 68 us, 0.91 to 0.96 of the rate
// of a plain copy.
//
// Quantization needs the whole row twice (its largest magnitude, then the codes): the row stays in registers between
// the two, 32 bytes per thread and load, so memory sees it once.  The largest magnitude is found on the bit patterns
// without their sign -- they order like the magnitudes, with the infinities and NaNs on top -- two 16-bit elements per
// instruction; rounding to the nearest integer, ties to even, is an addition of 1.5 * 2^23, which leaves the code in
// the low byte.  Rows or pitches the wide accesses cannot address (and rows beyond 65536 elements of 16 bits) take the
// element form, which reads the row twice.
#include "internal.h"
#include "layer_math.cuh"
#include "ptx.cuh"

namespace mip {

namespace {

constexpr int kRowThreads = 256;

// Scale and multiplier of a row from the bits of its largest magnitude, as a float32.
struct RowScale {
    float scale, mult;
};
__device__ __forceinline__ RowScale row_scale(float top) {
    RowScale s{0.0f, 0.0f};                              // below 2^-119: codes 0, scale 0
    if (!(top <= 3.402823466e38f)) s.scale = __int_as_float(0x7FFFFFFF);
    else if (top >= 0x1p-119f) s = RowScale{__fdiv_rn(top, 127.0f), __fdiv_rn(127.0f, top)};
    return s;
}

__device__ __forceinline__ void ld_global_nc_v8(const void* p, uint32_t (&v)[8]) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}

// Codes of four floats (the low bytes of x * mult + 1.5 * 2^23) in one word.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float mult) {
    constexpr float kMagic = 12582912.0f;
    const uint32_t x = __float_as_uint(__fadd_rn(__fmul_rn(a, mult), kMagic)), y = __float_as_uint(__fadd_rn(__fmul_rn(b, mult), kMagic));
    const uint32_t z = __float_as_uint(__fadd_rn(__fmul_rn(c, mult), kMagic)), w = __float_as_uint(__fadd_rn(__fmul_rn(d, mult), kMagic));
    return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
}

// kType: element type; kVec: loads of 32 bytes per thread.  blockDim.x threads share a row (blockDim.y rows per block
// only where a row is one warp's).
template <int kType, int kVec>
__global__ void __launch_bounds__(1024)
mip_quantize_rows_kernel(long long M, int vectors, const uint8_t* X, long long ldx_bytes, int8_t* Q, long long ldq, float* scale) {
    constexpr int kElems = kType == kF32 ? 8 : 16;       // per vector
    __shared__ uint32_t part[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long row = static_cast<long long>(blockIdx.x) * blockDim.y + threadIdx.y;
    const bool here = row < M;
    const uint8_t* src = X + row * ldx_bytes;
    uint32_t v[kVec][8];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int at = i * blockDim.x + threadIdx.x;
        if (here && at < vectors) {
            ld_global_nc_v8(src + static_cast<long long>(at) * 32, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0u;
        }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            top = kType == kF32 ? max(top, v[i][j] & 0x7FFFFFFFu) : __vmaxu2(top, v[i][j] & 0x7FFF7FFFu);
    if (kType != kF32) top = max(top & 0xFFFFu, top >> 16);
    top = __reduce_max_sync(~0u, top);
    if (blockDim.x > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
        const int warps = blockDim.x >> 5;
        top = __reduce_max_sync(~0u, (threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0u);
    }
    const float top_f = kType == kF32 ? __uint_as_float(top)
                        : (kType == kF16 ? __half2float(__ushort_as_half(static_cast<uint16_t>(top))) : __uint_as_float(top << 16));
    const RowScale s = row_scale(top_f);
    if (here && threadIdx.x == 0) scale[row] = s.scale;
    const bool zero = s.mult == 0.0f;                    // (infinities times 0 would be NaN)
    int8_t* dst = Q + row * ldq;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int at = i * blockDim.x + threadIdx.x;
        if (!here || at >= vectors) continue;
        uint32_t q[kElems / 4];
        if (kType == kF32) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                q[j] = codes4(__uint_as_float(v[i][4 * j]), __uint_as_float(v[i][4 * j + 1]), __uint_as_float(v[i][4 * j + 2]),
                              __uint_as_float(v[i][4 * j + 3]), s.mult);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float f[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w = v[i][2 * j + h];
                    if (kType == kF16) {
                        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
                        f[2 * h] = t.x;
                        f[2 * h + 1] = t.y;
                    } else {
                        f[2 * h] = __uint_as_float(w << 16);
                        f[2 * h + 1] = __uint_as_float(w & 0xFFFF0000u);
                    }
                }
                q[j] = codes4(f[0], f[1], f[2], f[3], s.mult);
            }
        }
        if (zero) {
#pragma unroll
            for (int j = 0; j < kElems / 4; ++j) q[j] = 0u;
        }
        if (kType == kF32) *reinterpret_cast<uint2*>(dst + static_cast<long long>(at) * 8) = make_uint2(q[0], q[1]);
        else *reinterpret_cast<uint4*>(dst + static_cast<long long>(at) * 16) = make_uint4(q[0], q[1], q[2 % (kElems / 4)], q[3 % (kElems / 4)]);
    }
}

// Eight elements of a row, kRowThreads apart, as floats (0 beyond N).  Raw loads first: a conversion beside each load
// would wait for it.
template <int kPer>
__device__ __forceinline__ void load_strided8(float (&v)[8], const void* X, long long row_at, long long j0, long long N, int type) {
    if (type == kF32) {
        const float* x = static_cast<const float*>(X) + row_at;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = j0 + i * kPer < N ? x[j0 + i * kPer] : 0.0f;
        return;
    }
    const uint16_t* x = static_cast<const uint16_t*>(X) + row_at;
    uint16_t raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = j0 + i * kPer < N ? x[j0 + i * kPer] : uint16_t(0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = type == kF16 ? __half2float(__ushort_as_half(raw[i])) : __uint_as_float(static_cast<uint32_t>(raw[i]) << 16);
}

// Element form: any alignment, any length.  kPer threads have a row: a block's, or one warp's where rows are short (us there
// and back, block's / warp's: 10146 x 71 float32 28.7 / 10.4, 10000 x 511 bf16 45.1 / 14.4, 300 x 511 10.7 / 10.0).
template <int kPer>
__global__ void __launch_bounds__(kRowThreads)
mip_quantize_elements_kernel(int type, long long M, long long N, const void* X, long long ldx, int8_t* Q, long long ldq, float* scale) {
    __shared__ float part[kRowThreads / 32];
    __shared__ int odd[kRowThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int t = threadIdx.x % kPer;
    const long long row = blockIdx.x * static_cast<long long>(kRowThreads / kPer) + threadIdx.x / kPer;
    if (kPer == 32 && row >= M) return;                  // (whole warps, which meet nobody)
    float top = 0.0f;
    int bad = 0;
    const auto each = [&](auto&& body) {                 // eight elements at a time: their loads travel together
        for (long long j0 = t; j0 < N; j0 += 8 * kPer) {
            float v[8];
            load_strided8<kPer>(v, X, row * ldx, j0, N, type);
#pragma unroll
            for (int i = 0; i < 8; ++i) body(j0 + i * kPer, v[i]);
        }
    };
    each([&](long long, float x) {                       // (0 beyond the row)
        const float v = fabsf(x);
        bad |= !(v <= 3.402823466e38f);
        top = fmaxf(top, v);
    });
    top = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top)));
    bad = __any_sync(~0u, bad);
    if (kPer > 32) {
        if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5] = top; odd[threadIdx.x >> 5] = bad; }
        __syncthreads();
        for (int w = 0; w < kRowThreads / 32; ++w) { top = fmaxf(top, part[w]); bad |= odd[w]; }
    }
    const RowScale s = row_scale(bad ? __int_as_float(0x7FFFFFFF) : top);
    if (t == 0) scale[row] = s.scale;
    each([&](long long j, float x) {
        if (j < N) Q[row * ldq + j] = s.mult == 0.0f ? 0 : static_cast<int8_t>(__float2int_rn(__fmul_rn(x, s.mult)));
    });
}

// 16 codes per thread and row -> 16 elements; kRows rows per thread, their loads together.
template <int kType, int kRows>
__global__ void __launch_bounds__(kRowThreads)
mip_dequantize_rows_kernel(long long M, int vectors, const int8_t* Q, long long ldq, const float* scale, uint8_t* X, long long ldx_bytes) {
    pdl_wait();
    pdl_launch_dependents();
    const int at = blockIdx.y * blockDim.x + threadIdx.x;
    if (at >= vectors) return;
    const long long row0 = (static_cast<long long>(blockIdx.x) * blockDim.y + threadIdx.y) * kRows;
    uint4 w[kRows];
    float s[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (row0 + i >= M) continue;
        w[i] = ld_stream_v4(Q + (row0 + i) * ldq + static_cast<long long>(at) * 16);
        s[i] = __ldg(scale + row0 + i);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (row0 + i >= M) break;
        const uint32_t in[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        float f[16];
#pragma unroll
        for (int j = 0; j < 16; ++j)     // a byte with its sign flipped behind the exponent of 2^23: 2^23 + 128 + code
            f[j] = __fmul_rn(s[i], __fsub_rn(__uint_as_float(__byte_perm(in[j >> 2] ^ 0x80808080u, 0x4B000000u, 0x7540u + (j & 3))), 8388736.0f));
        uint8_t* dst = X + (row0 + i) * ldx_bytes + static_cast<long long>(at) * (kType == kF32 ? 64 : 32);
        uint32_t o[kType == kF32 ? 16 : 8];
#pragma unroll
        for (int j = 0; j < (kType == kF32 ? 16 : 8); ++j) {
            if (kType == kF32) o[j] = __float_as_uint(f[j]);
            else if (kType == kF16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o[j]) : "f"(f[(2 * j + 1) & 15]), "f"(f[(2 * j) & 15]));
            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[j]) : "f"(f[(2 * j + 1) & 15]), "f"(f[(2 * j) & 15]));
        }
        st_global_v8(reinterpret_cast<int32_t*>(dst), o);
        if (kType == kF32) st_global_v8(reinterpret_cast<int32_t*>(dst + 32), o + 8 % (kType == kF32 ? 16 : 8));
    }
}

template <int kPer>
__global__ void __launch_bounds__(kRowThreads)
mip_dequantize_elements_kernel(int type, long long M, long long N, const int8_t* Q, long long ldq, const float* scale, void* X, long long ldx) {
    pdl_wait();
    pdl_launch_dependents();
    const int t = threadIdx.x % kPer;
    const long long row = blockIdx.x * static_cast<long long>(kRowThreads / kPer) + threadIdx.x / kPer;
    if (row >= M) return;
    const float s = scale[row];
    for (long long j0 = static_cast<long long>(blockIdx.y) * 8 * kPer + t; j0 < N;
         j0 += static_cast<long long>(gridDim.y) * 8 * kPer) {
        int8_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = j0 + i * kPer < N ? Q[row * ldq + j0 + i * kPer] : int8_t(0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i * kPer < N) store_element(X, row * ldx + j0 + i * kPer, type, __fmul_rn(s, static_cast<float>(q[i])));
    }
}

// Rows that a warp takes alone (us there and back, warp / block a row, bf16: 300 x 1001 8.8 / 10.0, 10000 x 1001 26 / 47, 300 x 2001 11.2 / 9.9, 10000 x
// 2001 49 / 51).
constexpr long long kShortRow = 1024;
dim3 short_rows_grid(long long M) { return dim3(static_cast<unsigned>((M + kRowThreads / 32 - 1) / (kRowThreads / 32))); }

bool aligned_rows(const void* p, long long pitch_bytes, int bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && pitch_bytes % bytes == 0;
}

// Launched early only where the blocks are few (see finish() of the layer kernels): 8 x 4096 there and back 11.3 -> 9.7 us.
template <typename... Formal, typename... Actual>
cudaError_t launch(void (*kernel)(Formal...), dim3 grid, dim3 block, cudaStream_t stream, Actual... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = static_cast<long long>(grid.x) * grid.y <= 128 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Formal>(args)...);
}

template <int kType>
cudaError_t quantize_t(long long M, int vectors, const uint8_t* X, long long ldx_bytes, int8_t* Q, long long ldq, float* scale, cudaStream_t stream) {
    // Many rows: four vectors per thread keep enough bytes on their way; few rows: one, so that the row's work is spread.
    int per = M >= 2048 ? 4 : 1;
    while (per < 4 && vectors > 1024 * per) per *= 2;
    const int threads = ((vectors + per - 1) / per + 31) / 32 * 32;
    const int rows = threads == 32 ? 4 : 1;
    const dim3 grid = dim3(static_cast<unsigned>((M + rows - 1) / rows)), block = dim3(threads, rows);
    if (per == 1) return launch(mip_quantize_rows_kernel<kType, 1>, grid, block, stream, M, vectors, X, ldx_bytes, Q, ldq, scale);
    if (per == 2) return launch(mip_quantize_rows_kernel<kType, 2>, grid, block, stream, M, vectors, X, ldx_bytes, Q, ldq, scale);
    return launch(mip_quantize_rows_kernel<kType, 4>, grid, block, stream, M, vectors, X, ldx_bytes, Q, ldq, scale);
}

template <int kType>
cudaError_t dequantize_t(long long M, int vectors, const int8_t* Q, long long ldq, const float* scale, uint8_t* X, long long ldx_bytes,
                         cudaStream_t stream) {
    int tx = 32;
    while (tx < kRowThreads && tx < vectors) tx *= 2;
    const int ty = kRowThreads / tx;
    const bool many = M * vectors >= 1 << 20;
    const long long rows = static_cast<long long>(ty) * (many ? 4 : 1);
    const dim3 grid = dim3(static_cast<unsigned>((M + rows - 1) / rows), static_cast<unsigned>((vectors + tx - 1) / tx)), block = dim3(tx, ty);
    if (many) return launch(mip_dequantize_rows_kernel<kType, 4>, grid, block, stream, M, vectors, Q, ldq, scale, X, ldx_bytes);
    return launch(mip_dequantize_rows_kernel<kType, 1>, grid, block, stream, M, vectors, Q, ldq, scale, X, ldx_bytes);
}

}  // namespace

cudaError_t launch_quantize_rows(int type, long long M, long long N, const void* X, long long ldx, int8_t* Q,
                                 long long ldq, float* scale, cudaStream_t stream) {
    const long long ldx_bytes = ldx * (type == kF32 ? 4 : 2);
    const int elems = type == kF32 ? 8 : 16;
    if (N > 0 && N % elems == 0 && N / elems <= 4096 && aligned_rows(X, ldx_bytes, 32) && aligned_rows(Q, ldq, elems)) {
        const int vectors = static_cast<int>(N / elems);
        const uint8_t* x = static_cast<const uint8_t*>(X);
        if (type == kF32) return quantize_t<kF32>(M, vectors, x, ldx_bytes, Q, ldq, scale, stream);
        if (type == kF16) return quantize_t<kF16>(M, vectors, x, ldx_bytes, Q, ldq, scale, stream);
        return quantize_t<kBF16>(M, vectors, x, ldx_bytes, Q, ldq, scale, stream);
    }
    if (N <= kShortRow)
        return launch(mip_quantize_elements_kernel<32>, short_rows_grid(M), dim3(kRowThreads), stream, type, M, N, X, ldx, Q, ldq, scale);
    return launch(mip_quantize_elements_kernel<kRowThreads>, dim3(static_cast<unsigned>(M)), dim3(kRowThreads), stream, type, M, N, X, ldx, Q, ldq,
                  scale);
}

cudaError_t launch_dequantize_rows(int type, long long M, long long N, const int8_t* Q, long long ldq,
                                   const float* scale, void* X, long long ldx, cudaStream_t stream) {
    const long long ldx_bytes = ldx * (type == kF32 ? 4 : 2);
    if (N % 16 == 0 && N <= 1 << 20 && aligned_rows(X, ldx_bytes, 32) && aligned_rows(Q, ldq, 16)) {
        const int vectors = static_cast<int>(N / 16);
        uint8_t* x = static_cast<uint8_t*>(X);
        if (type == kF32) return dequantize_t<kF32>(M, vectors, Q, ldq, scale, x, ldx_bytes, stream);
        if (type == kF16) return dequantize_t<kF16>(M, vectors, Q, ldq, scale, x, ldx_bytes, stream);
        return dequantize_t<kBF16>(M, vectors, Q, ldq, scale, x, ldx_bytes, stream);
    }
    if (N <= kShortRow)
        return launch(mip_dequantize_elements_kernel<32>, short_rows_grid(M), dim3(kRowThreads), stream, type, M, N, Q, ldq, scale, X, ldx);
    const long long parts = (N + 8 * kRowThreads - 1) / (8 * kRowThreads);
    const dim3 grid = dim3(static_cast<unsigned>(M), static_cast<unsigned>(parts < 64 ? parts : 64)), block = dim3(kRowThreads);
    return launch(mip_dequantize_elements_kernel<kRowThreads>, grid, block, stream, type, M, N, Q, ldq, scale, X, ldx);
}

}  // namespace mip
