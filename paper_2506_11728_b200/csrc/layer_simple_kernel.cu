// Simplest form of the 8-bit layer's operators: 16 x 16 outputs per block, one per thread, operands
// through shared memory.  Right for every size, order and alignment.
#include "internal.h"
#include "layer_math.cuh"

namespace mip {

namespace {

constexpr int kT = 16;

// One output of a layer operator from its exact sums.
__device__ void finish_element(const LayerArgs& a, long long i, long long j, int s0, int s1) {
    const float as = scale_at(a.a_scale, i);
    const float z0 = __int2float_rn(s0) * as * scale_at(a.b0_scale, j);
    with_activation(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
        if (a.op == kOpLinear) {
            float y = activation<kAct>(a.bias ? z0 + a.bias[j] : z0);
            if (a.R) y += load_element(a.R, i * a.ldr + j, a.type);
            store_element(a.C, i * a.ldc + j, a.type, y);
            return;
        }
        const float z1 = __int2float_rn(s1) * as * scale_at(a.b1_scale, j);
        if (a.op == kOpGated) {
            store_element(a.C, i * a.ldc + j, a.type, activation<kAct>(z0) * z1);
            return;
        }
        float value, slope;
        activation_slope<kAct>(z0, value, slope);
        const float d = load_element(a.R, i * a.ldr + j, a.type);
        store_element(a.C, i * a.ldc + j, a.type, d * z1 * slope);
        store_element(a.C2, i * a.ldc2 + j, a.type, d * value);
    });
}

__global__ void mip_layer_simple_kernel(const LayerArgs a) {
    __shared__ int ta[kT][kT + 1], tb0[kT][kT + 1], tb1[kT][kT + 1];
    const int x = threadIdx.x, y = threadIdx.y;
    const long long tiles_n = (a.N + kT - 1) / kT;
    const long long i0 = blockIdx.x / tiles_n * kT, j0 = blockIdx.x % tiles_n * kT;
    int s0 = 0, s1 = 0;
    for (long long k0 = 0; k0 < a.K; k0 += kT) {
        const long long k = k0 + x;
        const bool ka = k < a.K && i0 + y < a.M, kb = k < a.K && j0 + y < a.N;
        const long long ia = (i0 + y) * a.lda + k;
        ta[y][x] = !ka ? 0 : (a.a_unsigned ? static_cast<int>(static_cast<const uint8_t*>(a.A)[ia])
                                           : static_cast<int>(static_cast<const int8_t*>(a.A)[ia]));
        tb0[y][x] = kb ? a.B0[(j0 + y) * a.ldb0 + k] : 0;
        tb1[y][x] = kb && a.B1 ? a.B1[(j0 + y) * a.ldb1 + k] : 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            s0 += ta[y][t] * tb0[x][t];
            s1 += ta[y][t] * tb1[x][t];
        }
        __syncthreads();
    }
    if (i0 + y < a.M && j0 + x < a.N) finish_element(a, i0 + y, j0 + x, s0, s1);
}

__global__ void mip_product_simple_kernel(const ProductArgs a) {
    __shared__ float ta[kT][kT + 1], tb[kT][kT + 1];
    const int x = threadIdx.x, y = threadIdx.y;
    const long long tiles_n = (a.N + kT - 1) / kT;
    const long long i0 = blockIdx.x / tiles_n * kT, j0 = blockIdx.x % tiles_n * kT;
    const long long i = i0 + y, j = j0 + x;
    float s = 0.0f;
    for (long long k0 = 0; k0 < a.K; k0 += kT) {
        if (a.a_order) {   // thread (y, x) reads row k0 + y of A, column i0 + x
            const bool in = k0 + y < a.K && i0 + x < a.M;
            ta[x][y] = in ? load_element(a.A, (k0 + y) * a.lda + i0 + x, kBF16) : 0.0f;
        } else {
            const bool in = i < a.M && k0 + x < a.K;
            ta[y][x] = in ? load_element(a.A, i * a.lda + k0 + x, kBF16) : 0.0f;
        }
        const bool in = k0 + y < a.K && j < a.N;
        tb[y][x] = in ? __bfloat162float(__float2bfloat16_rn(scale_at(a.b_scale, k0 + y) * a.B[(k0 + y) * a.ldb + j])) : 0.0f;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kT; ++t) s += ta[y][t] * tb[t][x];
        __syncthreads();
    }
    if (i < a.M && j < a.N) {
        if (a.accumulate) s += load_element(a.C, i * a.ldc + j, a.type);
        store_element(a.C, i * a.ldc + j, a.type, s);
    }
}

}  // namespace

cudaError_t launch_layer_simple(const LayerArgs& a, cudaStream_t stream) {
    const long long blocks = ((a.M + kT - 1) / kT) * ((a.N + kT - 1) / kT);
    if (blocks > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
    mip_layer_simple_kernel<<<static_cast<unsigned>(blocks), dim3(kT, kT), 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_product_simple(const ProductArgs& a, cudaStream_t stream) {
    const long long blocks = ((a.M + kT - 1) / kT) * ((a.N + kT - 1) / kT);
    if (blocks > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
    mip_product_simple_kernel<<<static_cast<unsigned>(blocks), dim3(kT, kT), 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace mip
