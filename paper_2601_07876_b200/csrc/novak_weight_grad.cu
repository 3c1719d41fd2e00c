// Weight and bias gradient of a linear layer from the 8-bit form of its input:
//     dW[n, k] = sum_t dy[t, n] h[t, k],   db[n] = sum_t dy[t, n].
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;
// Rows added up one after another before they join the total: a sum over all rows in one
// chain loses digits with its length.
constexpr int kRun = 1024;

__device__ __forceinline__ float param_at(const void *p, int type, int64_t i)
{
    return type == NOVAK_TYPE_F32 ? static_cast<const float *>(p)[i]
                                  : to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ void store_param(void *p, int type, int64_t i, float v)
{
    if (type == NOVAK_TYPE_F32) static_cast<float *>(p)[i] = v;
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// A 64 x 64 tile per CTA, 4 x 4 products per thread, in fp32.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) novak_weight_grad_plain_kernel(WeightGradArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float sdy[kDepth][kTile], sx[kDepth][kTile];
    const int64_t pitch = (a.n_in + 31) / 32 * 32;
    const int64_t n0 = static_cast<int64_t>(blockIdx.y) * kTile, k0 = static_cast<int64_t>(blockIdx.x) * kTile;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float acc[4][4] = {}, sum[4] = {};                  // of the last kRun rows
    float total[4][4] = {}, total_sum[4] = {};
    for (int64_t t0 = 0; t0 < a.rows; t0 += kDepth) {
        for (int i = threadIdx.x; i < kDepth * kTile; i += kThreads) {
            const int64_t t = t0 + i / kTile, n = n0 + i % kTile;
            sdy[i / kTile][i % kTile] = t < a.rows && n < a.n_out
                                            ? to_float(static_cast<const T *>(a.dy.ptr)[t * a.dy.stride + n]) : 0.0f;
        }
        if (threadIdx.x < kDepth * kTile / 8) {
            const int64_t t = t0 + threadIdx.x / 8, k = k0 + threadIdx.x % 8 * 8;
            float v[8] = {};
            if (t < a.rows && k < pitch)
                dequantize8(*reinterpret_cast<const uint2 *>(a.codes.codes + t * pitch + k),
                            a.codes.exps[(t * pitch + k) >> 5], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sx[threadIdx.x / 8][threadIdx.x % 8 * 8 + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = sdy[d][ty * 4 + i];
                x[i] = sx[d][tx + 16 * i];
                sum[i] += y[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(y[i], x[j], acc[i][j]);
        }
        __syncthreads();
        if ((t0 + kDepth) % kRun == 0 || t0 + kDepth >= a.rows) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    total[i][j] += acc[i][j];
                    acc[i][j] = 0.0f;
                }
                total_sum[i] += sum[i];
                sum[i] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + ty * 4 + i;
        if (n >= a.n_out) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t k = k0 + tx + 16 * j;
            if (k >= a.n_in) continue;
            float v = total[i][j];
            // h = xhat w + b: w sum(dy xhat) + b sum(dy)
            if (a.weight)
                v = fmaf(v, param_at(a.weight, a.param_type, k), param_at(a.bias, a.param_type, k) * total_sum[i]);
            store_param(a.dw, a.grad_type, n * a.n_in + k, v);
        }
        if (a.db && blockIdx.x == 0 && tx == 0) store_param(a.db, a.grad_type, n, total_sum[i]);
    }
}

}  // namespace

size_t weight_grad_bytes(const Mat &, int, int64_t, int64_t, int64_t) { return 0; }

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t stream)
{
    const dim3 grid(static_cast<unsigned>((a.n_in + kTile - 1) / kTile),
                    static_cast<unsigned>((a.n_out + kTile - 1) / kTile));
    if (a.type == NOVAK_TYPE_F32) novak_weight_grad_plain_kernel<0><<<grid, kThreads, 0, stream>>>(a);
    else novak_weight_grad_plain_kernel<1><<<grid, kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace novak
