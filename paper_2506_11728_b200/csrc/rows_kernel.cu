// Rows of activations to 8-bit codes with one scale each, and back.
#include "internal.h"
#include "layer_math.cuh"

namespace mip {

namespace {

constexpr int kRowThreads = 256;

__global__ void mip_quantize_rows_kernel(int type, long long N, const void* X, long long ldx, int8_t* Q, long long ldq,
                                         float* scale) {
    __shared__ float part[kRowThreads / 32];
    __shared__ int odd[kRowThreads / 32];
    const long long row = blockIdx.x;
    float top = 0.0f;
    int bad = 0;
    for (long long j = threadIdx.x; j < N; j += kRowThreads) {
        const float v = fabsf(load_element(X, row * ldx + j, type));
        bad |= !(v <= 3.402823466e38f);
        top = fmaxf(top, v);
    }
    for (int d = 16; d; d >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        bad |= __shfl_xor_sync(~0u, bad, d);
    }
    if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5] = top; odd[threadIdx.x >> 5] = bad; }
    __syncthreads();
    for (int w = 0; w < kRowThreads / 32; ++w) { top = fmaxf(top, part[w]); bad |= odd[w]; }
    const bool zero = bad || top < 0x1p-119f;
    const float r = zero ? 0.0f : __fdiv_rn(127.0f, top);
    if (threadIdx.x == 0) scale[row] = bad ? __int_as_float(0x7FFFFFFF) : (zero ? 0.0f : __fdiv_rn(top, 127.0f));
    for (long long j = threadIdx.x; j < N; j += kRowThreads)
        Q[row * ldq + j] = zero ? 0 : static_cast<int8_t>(__float2int_rn(__fmul_rn(load_element(X, row * ldx + j, type), r)));
}

__global__ void mip_dequantize_rows_kernel(int type, long long N, const int8_t* Q, long long ldq, const float* scale,
                                           void* X, long long ldx) {
    const long long row = blockIdx.x;
    const float s = scale[row];
    for (long long j = threadIdx.x; j < N; j += kRowThreads)
        store_element(X, row * ldx + j, type, __fmul_rn(s, static_cast<float>(Q[row * ldq + j])));
}

}  // namespace

cudaError_t launch_quantize_rows(int type, long long M, long long N, const void* X, long long ldx, int8_t* Q,
                                 long long ldq, float* scale, cudaStream_t stream) {
    mip_quantize_rows_kernel<<<static_cast<unsigned>(M), kRowThreads, 0, stream>>>(type, N, X, ldx, Q, ldq, scale);
    return cudaGetLastError();
}

cudaError_t launch_dequantize_rows(int type, long long M, long long N, const int8_t* Q, long long ldq,
                                   const float* scale, void* X, long long ldx, cudaStream_t stream) {
    mip_dequantize_rows_kernel<<<static_cast<unsigned>(M), kRowThreads, 0, stream>>>(type, N, Q, ldq, scale, X, ldx);
    return cudaGetLastError();
}

}  // namespace mip
