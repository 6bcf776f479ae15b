// The transforms of the 8-bit layer on their own: adds planes of partial sums that a dense kernel left behind when its
// K was split over the grid, and finishes them.  Bound by the planes' bytes, which the L2 still holds (1024 x 1024
// float32 in 4 parts: 5 us, half of it the launch).  With no planes
// every sum is 0: the case K == 0.
#include "internal.h"
#include "layer_math.cuh"

namespace mip {

namespace {

constexpr int kThreads = 256;
constexpr int kCols = 4;             // columns per thread: one 16-byte read per plane

template <int kOp>
__global__ void __launch_bounds__(kThreads)
mip_layer_finish_kernel(const LayerArgs a, const PartialPlanes s) {
    const long long row = static_cast<long long>(blockIdx.y) * blockDim.y + threadIdx.y;
    const long long col = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) * kCols;
    if (row >= a.M || col >= a.N) return;
    int s0[kCols] = {0, 0, 0, 0}, s1[kCols] = {0, 0, 0, 0};
    const int* src = static_cast<const int*>(s.base) + row * s.pitch + col;
#pragma unroll 4
    for (int k = 0; k < s.split; ++k) {
        const int4 x = *reinterpret_cast<const int4*>(src + k * s.plane_rows * s.pitch);
        s0[0] += x.x; s0[1] += x.y; s0[2] += x.z; s0[3] += x.w;
        if (kOp != kOpLinear) {
            const int4 y = *reinterpret_cast<const int4*>(src + k * s.plane_rows * s.pitch + s.second);
            s1[0] += y.x; s1[1] += y.y; s1[2] += y.z; s1[3] += y.w;
        }
    }
    const float as = scale_at(a.a_scale, row);
    const int cols = static_cast<int>(min(static_cast<long long>(kCols), a.N - col));
    float r[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) r[j] = (kOp != kOpGated && a.R && j < cols) ? load_element(a.R, row * a.ldr + col + j, a.type) : 0.0f;
    with_activation(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            if (j >= cols) break;
            const float z0 = __int2float_rn(s0[j]) * as * scale_at(a.b0_scale, col + j);
            const long long at = row * a.ldc + col + j;
            if (kOp == kOpLinear) {
                store_element(a.C, at, a.type, activation<kAct>(z0 + (a.bias ? __ldg(a.bias + col + j) : 0.0f)) + r[j]);
            } else {
                const float z1 = __int2float_rn(s1[j]) * as * scale_at(a.b1_scale, col + j);
                if (kOp == kOpGated) {
                    store_element(a.C, at, a.type, activation<kAct>(z0) * z1);
                } else {
                    float value, slope;
                    activation_slope<kAct>(z0, value, slope);
                    store_element(a.C, at, a.type, r[j] * z1 * slope);
                    store_element(a.C2, row * a.ldc2 + col + j, a.type, r[j] * value);
                }
            }
        }
    });
}

__global__ void __launch_bounds__(kThreads)
mip_product_finish_kernel(const ProductArgs a, const PartialPlanes s) {
    const long long row = static_cast<long long>(blockIdx.y) * blockDim.y + threadIdx.y;
    const long long col = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) * kCols;
    if (row >= a.M || col >= a.N) return;
    float v[kCols] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float* src = static_cast<const float*>(s.base) + row * s.pitch + col;
#pragma unroll 4
    for (int k = 0; k < s.split; ++k) {              // in the order of K: the result does not depend on the run
        const float4 x = *reinterpret_cast<const float4*>(src + k * s.plane_rows * s.pitch);
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
    const int cols = static_cast<int>(min(static_cast<long long>(kCols), a.N - col));
#pragma unroll
    for (int j = 0; j < kCols; ++j)
        if (a.accumulate && j < cols) v[j] += load_element(a.C, row * a.ldc + col + j, a.type);
#pragma unroll
    for (int j = 0; j < kCols; ++j)
        if (j < cols) store_element(a.C, row * a.ldc + col + j, a.type, v[j]);
}

// These kernels are launched in order (no programmatic stream serialisation): they have nothing to do before the kernel in
// front of them is over, and as many small blocks they would sit on the SMs until then.
template <typename Args>
cudaError_t finish(void (*kernel)(const Args, const PartialPlanes), const Args& a, const PartialPlanes& s, cudaStream_t stream) {
    int tx = 8;
    while (tx < kThreads && tx * kCols < a.N) tx *= 2;
    const int ty = kThreads / tx;
    // (the rows go in launches of at most 65535 blocks, the limit of the grid's second dimension)
    const long long step = 65535LL * ty;
    for (long long row = 0; row < a.M; row += step) {
        Args part = a;
        PartialPlanes planes = s;
        part.M = a.M - row < step ? a.M - row : step;
        part.advance(row);
        if (s.base) planes.base = static_cast<const char*>(s.base) + row * s.pitch * 4;
        const dim3 grid(static_cast<unsigned>((a.N + tx * kCols - 1) / (tx * kCols)), static_cast<unsigned>((part.M + ty - 1) / ty));
        kernel<<<grid, dim3(tx, ty), 0, stream>>>(part, planes);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_layer_finish(const LayerArgs& a, const PartialPlanes& s, cudaStream_t stream) {
    if (a.op == kOpLinear) return finish(mip_layer_finish_kernel<kOpLinear>, a, s, stream);
    if (a.op == kOpGated) return finish(mip_layer_finish_kernel<kOpGated>, a, s, stream);
    return finish(mip_layer_finish_kernel<kOpGatedGrad>, a, s, stream);
}

cudaError_t launch_product_finish(const ProductArgs& a, const PartialPlanes& s, cudaStream_t stream) {
    return finish(mip_product_finish_kernel, a, s, stream);
}

}  // namespace mip
