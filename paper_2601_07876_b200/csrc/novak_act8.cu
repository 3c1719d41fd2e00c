// The 8-bit form of activations (packing, unpacking) and the activation
// functions that leave it and take it up.  One element costs one read and one
// write of everything it has: HBM-bound.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;
constexpr int kIdentity = -1;

template <int KIND>
__device__ __forceinline__ float act(float u)
{
    if constexpr (KIND == NOVAK_ACT_GELU) return 0.5f * u * erfcf(-u * 0.70710678f);
    if constexpr (KIND == NOVAK_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 is the logistic function of 2 z
        const float z2 = 1.5957691f * fmaf(0.044715f * u * u, u, u);
        return u / (1.0f + expf(-z2));
    }
    if constexpr (KIND == NOVAK_ACT_SILU) return u / (1.0f + expf(-u));
    return u;
}

template <int KIND>
__device__ __forceinline__ float act_slope(float u)
{
    if constexpr (KIND == NOVAK_ACT_GELU)
        return fmaf(u * 0.39894228f, expf(-0.5f * u * u), 0.5f * erfcf(-u * 0.70710678f));
    if constexpr (KIND == NOVAK_ACT_GELU_TANH) {
        const float p = 1.0f / (1.0f + expf(-1.5957691f * fmaf(0.044715f * u * u, u, u)));
        // p is 0 or 1 long before |u| = 30; beyond, u^2 must not become the infinity of 0 * inf
        const float t = fminf(fmaxf(u, -30.0f), 30.0f);
        return p * (1.0f + t * (1.0f - p) * 1.5957691f * fmaf(3.0f * 0.044715f, t * t, 1.0f));
    }
    if constexpr (KIND == NOVAK_ACT_SILU) {
        const float p = 1.0f / (1.0f + expf(-u));
        return p * fmaf(u, 1.0f - p, 1.0f);
    }
    return 1.0f;
}

// One thread, eight elements; four threads share a block.  A row has pitch / 8
// groups, a multiple of four, so a quad never straddles rows.
template <int KIND, int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads)
novak_activation_kernel(const typename Elem<TYPE>::T *u, int64_t u_stride, typename Elem<TYPE>::T *a,
                        int64_t a_stride, Codes uc, Codes ac, int64_t rows, int64_t cols)
{
    using T = typename Elem<TYPE>::T;
    const int64_t per_row = (cols + 31) / 32 * 4, n = rows * per_row;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
    // (n is a multiple of 4 and so is the first index of a quad: it stays together)
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i - (threadIdx.x & 31) < n; i += step) {
        const bool live = i < n;
        const int64_t row = live ? i / per_row : 0, col = live ? (i - row * per_row) * 8 : 0;
        float v[8], f[8];
        load8<WIDE>(u + row * u_stride, col, live ? cols : 0, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = to_float(from_float<T>(act<KIND>(v[k])));
        uint32_t exp;
        if (uc.codes) {
            const uint2 q = quantize8(v, exp);
            if (live) {
                reinterpret_cast<uint2 *>(uc.codes)[i] = q;
                if ((i & 3) == 0) uc.exps[i >> 2] = static_cast<uint8_t>(exp);
            }
        }
        if (ac.codes) {
            const uint2 q = quantize8(f, exp);
            if (live) {
                reinterpret_cast<uint2 *>(ac.codes)[i] = q;
                if ((i & 3) == 0) ac.exps[i >> 2] = static_cast<uint8_t>(exp);
            }
        }
        if (a && live) store8<WIDE>(a + row * a_stride, col, cols, f);
    }
}

template <int KIND, int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads)
novak_activation_backward_kernel(const typename Elem<TYPE>::T *da, int64_t da_stride,
                                 const typename Elem<TYPE>::T *u, int64_t u_stride, Codes uc,
                                 typename Elem<TYPE>::T *du, int64_t du_stride, int64_t rows, int64_t cols)
{
    const int64_t per_row = (cols + 31) / 32 * 4, n = rows * per_row;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += step) {
        const int64_t row = i / per_row, col = (i - row * per_row) * 8;
        float v[8], g[8];
        if (uc.codes) dequantize8(reinterpret_cast<const uint2 *>(uc.codes)[i], uc.exps[i >> 2], v);
        else load8<WIDE>(u + row * u_stride, col, cols, v);
        if constexpr (KIND != kIdentity) {
            load8<WIDE>(da + row * da_stride, col, cols, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = g[k] * act_slope<KIND>(v[k]);
        }
        store8<WIDE>(du + row * du_stride, col, cols, v);
    }
}

int grid_for(int64_t rows, int64_t cols)
{
    const int64_t n = rows * (act_pitch(cols) / 8);
    return static_cast<int>(std::min<int64_t>((n + kThreads - 1) / kThreads, 148 * 64));
}

template <int KIND, int TYPE>
cudaError_t forward(Mat u, Mat a, Codes uc, Codes ac, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    const int grid = grid_for(rows, cols);
    const bool w = wide(u, TYPE, rows) && (!a.ptr || wide(a, TYPE, rows));
    auto kernel = w ? novak_activation_kernel<KIND, TYPE, true> : novak_activation_kernel<KIND, TYPE, false>;
    kernel<<<grid, kThreads, 0, stream>>>(static_cast<const T *>(u.ptr), u.stride, static_cast<T *>(a.ptr),
                                          a.stride, uc, ac, rows, cols);
    return cudaGetLastError();
}

template <int KIND, int TYPE>
cudaError_t backward(Mat da, Mat u, Codes uc, Mat du, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    const int grid = grid_for(rows, cols);
    const bool w = (!da.ptr || wide(da, TYPE, rows)) && (!u.ptr || wide(u, TYPE, rows)) && wide(du, TYPE, rows);
    auto kernel = w ? novak_activation_backward_kernel<KIND, TYPE, true>
                    : novak_activation_backward_kernel<KIND, TYPE, false>;
    kernel<<<grid, kThreads, 0, stream>>>(static_cast<const T *>(da.ptr), da.stride,
                                          static_cast<const T *>(u.ptr), u.stride, uc,
                                          static_cast<T *>(du.ptr), du.stride, rows, cols);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_activation(Mat u, Mat a, int type, int kind, Codes uc, Codes ac, int64_t rows,
                              int64_t cols, cudaStream_t stream)
{
#define NOVAK_CASE(K)                                                                             \
    case K:                                                                                       \
        return type == NOVAK_TYPE_F32 ? forward<K, NOVAK_TYPE_F32>(u, a, uc, ac, rows, cols, stream) \
                                      : forward<K, NOVAK_TYPE_BF16>(u, a, uc, ac, rows, cols, stream)
    switch (kind) {
        NOVAK_CASE(NOVAK_ACT_GELU);
        NOVAK_CASE(NOVAK_ACT_GELU_TANH);
        NOVAK_CASE(NOVAK_ACT_SILU);
        NOVAK_CASE(kIdentity);
    }
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

cudaError_t launch_activation_backward(Mat da, Mat u, int type, int kind, Codes uc, Mat du, int64_t rows,
                                       int64_t cols, cudaStream_t stream)
{
#define NOVAK_CASE(K)                                                                          \
    case K:                                                                                    \
        return type == NOVAK_TYPE_F32 ? backward<K, NOVAK_TYPE_F32>(da, u, uc, du, rows, cols, stream) \
                                      : backward<K, NOVAK_TYPE_BF16>(da, u, uc, du, rows, cols, stream)
    switch (kind) {
        NOVAK_CASE(NOVAK_ACT_GELU);
        NOVAK_CASE(NOVAK_ACT_GELU_TANH);
        NOVAK_CASE(NOVAK_ACT_SILU);
        NOVAK_CASE(kIdentity);
    }
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

}  // namespace novak
