// Layer norm, forward and backward.
//     mean = sum(x)/C, rstd = 1/sqrt(sum((x - mean)^2)/C + eps), xhat = (x - mean) rstd,
//     y = xhat w + b;
//     g = dy w, dx = rstd (g - sum(g)/C - xhat sum(g xhat)/C),
//     dw = sum over rows of dy xhat, db = sum over rows of dy.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;
constexpr int kSplitRows = 128;      // rows per partial sum of a column
constexpr int kColsPerCta = 32;

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

// One CTA per row, any length: the row is read three times (from L2 after the
// first time).
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_layer_norm_long_kernel(NormArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[33];
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const float inv_cols = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x.ptr) + row * a.x.stride;
        T *y = static_cast<T *>(a.y.ptr) + row * a.y.stride;
        float sum = 0.0f, v[8];
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(x, c, a.cols, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
        const float mean = block_sum(sum, scratch) * inv_cols;
        float sq = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(x, c, a.cols, v);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < a.cols) sq = fmaf(v[k] - mean, v[k] - mean, sq);
        }
        const float rstd = 1.0f / sqrtf(fmaf(block_sum(sq, scratch), inv_cols, a.eps));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        // (the pitch is a multiple of 32: a quad is inside it, or outside, as a whole)
        for (int64_t c0 = 0; c0 < pitch; c0 += kThreads * 8) {
            const int64_t c = c0 + threadIdx.x * 8;
            load8<WIDE>(x, c, a.cols, v);
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool in = c + k < a.cols;
                v[k] = in ? (v[k] - mean) * rstd : 0.0f;
                o[k] = in ? fmaf(v[k], param_at(a.weight, a.param_type, c + k),
                                 a.bias ? param_at(a.bias, a.param_type, c + k) : 0.0f) : 0.0f;
            }
            store8<WIDE>(y, c, a.cols, o);
            if (a.codes.codes) {
                uint32_t exp;
                const uint2 q = quantize8(v, exp);
                if (c < pitch) {
                    *reinterpret_cast<uint2 *>(a.codes.codes + row * pitch + c) = q;
                    if ((threadIdx.x & 3) == 0) a.codes.exps[(row * pitch + c) >> 5] = static_cast<uint8_t>(exp);
                }
            }
        }
    }
}

// xhat of eight elements, from the 8-bit form or from x.
template <int TYPE, bool WIDE>
__device__ __forceinline__ void xhat8(const NormBackArgs &a, int64_t row, int64_t c, int64_t pitch, float mean,
                                      float rstd, float (&v)[8])
{
    if (a.codes.codes) {
        dequantize8(*reinterpret_cast<const uint2 *>(a.codes.codes + row * pitch + c),
                    a.codes.exps[(row * pitch + c) >> 5], v);
    } else {
        using T = typename Elem<TYPE>::T;
        load8<WIDE>(static_cast<const T *>(a.x.ptr) + row * a.x.stride, c, a.cols, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < a.cols ? (v[k] - mean) * rstd : 0.0f;
    }
}

template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_layer_norm_back_long_kernel(NormBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[33];
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const float inv_cols = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dy.ptr) + row * a.dy.stride;
        T *dx = static_cast<T *>(a.dx.ptr) + row * a.dx.stride;
        const float rstd = a.rstd[row], mean = a.mean ? a.mean[row] : 0.0f;
        float s1 = 0.0f, s2 = 0.0f, g[8], xh[8];
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(dy, c, a.cols, g);
            xhat8<TYPE, WIDE>(a, row, c, pitch, mean, rstd, xh);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < a.cols) {
                    g[k] *= param_at(a.weight, a.param_type, c + k);
                    s1 += g[k];
                    s2 = fmaf(g[k], xh[k], s2);
                }
        }
        s1 = block_sum(s1, scratch) * inv_cols;
        s2 = block_sum(s2, scratch) * inv_cols;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(dy, c, a.cols, g);
            xhat8<TYPE, WIDE>(a, row, c, pitch, mean, rstd, xh);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < a.cols)
                    g[k] = rstd * (fmaf(-xh[k], s2, g[k] * param_at(a.weight, a.param_type, c + k)) - s1);
            store8<WIDE>(dx, c, a.cols, g);
        }
    }
}

// Column sums of dy xhat and dy over kSplitRows rows at a time: 32 columns per
// CTA, partial[split][2][cols].
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_layer_norm_columns_kernel(NormBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float part[2][kThreads / 4][kColsPerCta + 1];
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const int quad = threadIdx.x & 3, lane = threadIdx.x >> 2;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kColsPerCta + quad * 8;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kSplitRows;
    const int64_t row1 = min(row0 + kSplitRows, a.rows);
    float dw[8] = {}, db[8] = {}, g[8], xh[8];
    for (int64_t row = row0 + lane; row < row1; row += kThreads / 4) {
        load8<WIDE>(static_cast<const T *>(a.dy.ptr) + row * a.dy.stride, c, a.cols, g);
        xhat8<TYPE, WIDE>(a, row, c, pitch, a.mean ? a.mean[row] : 0.0f, a.rstd[row], xh);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < a.cols) {
                dw[k] = fmaf(g[k], xh[k], dw[k]);
                db[k] += g[k];
            }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        part[0][lane][quad * 8 + k] = dw[k];
        part[1][lane][quad * 8 + k] = db[k];
    }
    __syncthreads();
    if (threadIdx.x < 2 * kColsPerCta) {
        const int which = threadIdx.x / kColsPerCta, col = threadIdx.x % kColsPerCta;
        float s = 0.0f;
        for (int i = 0; i < kThreads / 4; ++i) s += part[which][i][col];
        const int64_t out = static_cast<int64_t>(blockIdx.x) * kColsPerCta + col;
        if (out < a.cols) a.work[(static_cast<int64_t>(blockIdx.y) * 2 + which) * a.cols + out] = s;
    }
}

// dw, db from the partial sums, in order.
__global__ void __launch_bounds__(kThreads)
novak_layer_norm_finish_kernel(const float *work, int64_t splits, int64_t cols, void *dweight, void *dbias, int type)
{
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= cols) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t s = 0; s < splits; ++s) {
        dw += work[(2 * s) * cols + c];
        db += work[(2 * s + 1) * cols + c];
    }
    if (dweight) store_param(dweight, type, c, dw);
    if (dbias) store_param(dbias, type, c, db);
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.x, a.type, a.rows) && wide(a.y, a.type, a.rows);
    const int grid = static_cast<int>(std::min<int64_t>(a.rows, 148 * 8));
    auto kernel = a.type == NOVAK_TYPE_F32
                      ? (w ? novak_layer_norm_long_kernel<0, true> : novak_layer_norm_long_kernel<0, false>)
                      : (w ? novak_layer_norm_long_kernel<1, true> : novak_layer_norm_long_kernel<1, false>);
    kernel<<<grid, kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

size_t layer_norm_backward_bytes(int64_t rows, int64_t cols)
{
    return static_cast<size_t>((rows + kSplitRows - 1) / kSplitRows * 2 * cols) * sizeof(float);
}

cudaError_t launch_layer_norm_backward(const NormBackArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.dy, a.type, a.rows) && wide(a.dx, a.type, a.rows) &&
                   (!a.x.ptr || wide(a.x, a.type, a.rows));
    const int64_t splits = (a.rows + kSplitRows - 1) / kSplitRows;
    const int t = a.type == NOVAK_TYPE_F32 ? 0 : 1;
    if (a.rows > 0 && (a.dweight || a.dbias)) {
        auto columns = t == 0 ? (w ? novak_layer_norm_columns_kernel<0, true> : novak_layer_norm_columns_kernel<0, false>)
                              : (w ? novak_layer_norm_columns_kernel<1, true> : novak_layer_norm_columns_kernel<1, false>);
        const dim3 grid(static_cast<unsigned>((a.cols + kColsPerCta - 1) / kColsPerCta), static_cast<unsigned>(splits));
        columns<<<grid, kThreads, 0, stream>>>(a);
    }
    if (a.rows > 0) {
        auto kernel = t == 0 ? (w ? novak_layer_norm_back_long_kernel<0, true> : novak_layer_norm_back_long_kernel<0, false>)
                             : (w ? novak_layer_norm_back_long_kernel<1, true> : novak_layer_norm_back_long_kernel<1, false>);
        kernel<<<static_cast<int>(std::min<int64_t>(a.rows, 148 * 8)), kThreads, 0, stream>>>(a);
    }
    if (a.dweight || a.dbias)
        novak_layer_norm_finish_kernel<<<static_cast<unsigned>((a.cols + kThreads - 1) / kThreads), kThreads, 0, stream>>>(
            a.work, splits, a.cols, a.dweight, a.dbias, a.grad_type);
    return cudaGetLastError();
}

}  // namespace novak
