// The 8-bit form of activations (packing, unpacking) and the activation functions
// that leave it and take it up.  One element costs one read and one write of
// everything it has: HBM-bound.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;
constexpr int kIdentity = -1;
constexpr int kUnroll = 2;          // groups of 8 per thread, all loads first
constexpr int kNarrowUnroll = 8;    // elements per thread where rows are not aligned

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ F2 exp2_approx(F2 x) { return F2(exp2_approx(x.lo()), exp2_approx(x.hi())); }
__device__ __forceinline__ F2 rcp_approx(F2 x) { return F2(rcp_approx(x.lo()), rcp_approx(x.hi())); }

// Phi(-|u|) and exp(-u^2/2), Phi the normal distribution function, by formula
// 7.1.26 of Abramowitz and Stegun (erf to 1.5e-7) for x = |u| / sqrt(2).
__device__ __forceinline__ void normal_tail(F2 u, F2 &mag, F2 &tail, F2 &e)
{
    mag = F2(fabsf(u.lo()), fabsf(u.hi()));
    const F2 t = rcp_approx(fma2(mag, F2(0.3275911f * 0.70710678f), F2(1.0f)));
    e = exp2_approx(u * u * F2(-0.5f * 1.44269504f));
    F2 p = fma2(t, F2(0.5f * 1.061405429f), F2(0.5f * -1.453152027f));
    p = fma2(p, t, F2(0.5f * 1.421413741f));
    p = fma2(p, t, F2(0.5f * -0.284496736f));
    p = fma2(p, t, F2(0.5f * 0.254829592f));
    tail = p * t * e;
}

// (1 + tanh z) / 2 is the logistic function of 2 z: tanh-GELU is u times it.
constexpr float kTanh = 1.5957691216f, kCubic = 0.044715f, kLog2e = 1.44269504f;

__device__ __forceinline__ F2 logistic(F2 minus_log2e_z)
{
    return rcp_approx(exp2_approx(minus_log2e_z) + F2(1.0f));
}
__device__ __forceinline__ F2 tanh_argument(F2 u)
{
    return u * fma2(u * u, F2(-kLog2e * kTanh * kCubic), F2(-kLog2e * kTanh));
}

template <int KIND>
__device__ __forceinline__ F2 act(F2 u)
{
    if constexpr (KIND == NOVAK_ACT_GELU) {
        F2 mag, tail, e;
        normal_tail(u, mag, tail, e);
        // u (1 - tail) above zero, u tail below
        return fma2(mag * F2(-1.0f), tail, F2(fmaxf(u.lo(), 0.0f), fmaxf(u.hi(), 0.0f)));
    }
    if constexpr (KIND == NOVAK_ACT_GELU_TANH) return u * logistic(tanh_argument(u));
    if constexpr (KIND == NOVAK_ACT_SILU) return u * logistic(u * F2(-kLog2e));
    return u;
}

template <int KIND>
__device__ __forceinline__ F2 act_slope(F2 u)
{
    if constexpr (KIND == NOVAK_ACT_GELU) {
        F2 mag, tail, e;
        normal_tail(u, mag, tail, e);
        const F2 h = fma2(tail, F2(-1.0f), F2(0.5f));       // Phi(u) = 1/2 +- h
        const F2 phi = F2(copysignf(h.lo(), u.lo()), copysignf(h.hi(), u.hi())) + F2(0.5f);
        return fma2(u * F2(0.39894228f), e, phi);
    }
    if constexpr (KIND == NOVAK_ACT_GELU_TANH) {
        const F2 p = logistic(tanh_argument(u));
        // p is 0 or 1 long before |u| = 30; beyond, u^2 must not become the infinity of 0 * inf
        const F2 t(fminf(fmaxf(u.lo(), -30.0f), 30.0f), fminf(fmaxf(u.hi(), -30.0f), 30.0f));
        const F2 slope = t * fma2(t * t, F2(3.0f * kCubic * kTanh), F2(kTanh));
        return p * fma2(fma2(p, F2(-1.0f), F2(1.0f)), slope, F2(1.0f));
    }
    if constexpr (KIND == NOVAK_ACT_SILU) {
        const F2 p = logistic(u * F2(-kLog2e));
        return p * fma2(fma2(p, F2(-1.0f), F2(1.0f)), u, F2(1.0f));
    }
    return F2(1.0f);
}

// Where a thread's elements are.  FLAT: rows without gaps, a multiple of 32 long, are
// one run of elements.  Otherwise 2^log2 neighbouring threads share a row.
struct Place {
    int64_t rows, cols;
    int64_t groups;         // of V elements: all of them (FLAT), or of a row's pitch
    int log2;
};

struct At {
    int64_t row, col;       // FLAT: row 0, col over the whole run
    bool in;                // inside the rows and their padding
};

template <bool FLAT, int V, int UNROLL>
__device__ __forceinline__ At place(const Place &p, int64_t first_row, int u)
{
    if constexpr (FLAT) {
        const int64_t g = (static_cast<int64_t>(blockIdx.x) * UNROLL + u) * kThreads + threadIdx.x;
        return {0, g * V, g < p.groups};
    } else {
        const int64_t g = (static_cast<int64_t>(blockIdx.x) << p.log2) + (threadIdx.x & ((1 << p.log2) - 1));
        const int64_t row = first_row + (static_cast<int64_t>(u) << (8 - p.log2)) + (threadIdx.x >> p.log2);
        return {row, g * V, g < p.groups && row < p.rows};
    }
}

template <bool FLAT> __device__ __forceinline__ int64_t code_at(const Place &p, const At &at, int64_t pitch)
{
    return FLAT ? at.col : at.row * pitch + at.col;
}

__device__ __forceinline__ void put(const Codes &c, int64_t at, bool in, const F2 (&v)[4], uint32_t top)
{
    uint32_t exp;
    const uint2 q = quantize8(v, top, exp);
    if (in) {
        *reinterpret_cast<uint2 *>(c.codes + at) = q;
        if ((threadIdx.x & 3) == 0) c.exps[at >> 5] = static_cast<uint8_t>(exp);
    }
}

// One thread, eight elements at a time; a quad of threads has a block.
template <int KIND, int TYPE, bool FLAT>
__global__ void __launch_bounds__(kThreads)
novak_activation_kernel(const typename Elem<TYPE>::T *u, int64_t u_stride, typename Elem<TYPE>::T *a, int64_t a_stride,
                        Codes uc, Codes ac, Place p)
{
    const int64_t pitch = (p.cols + 31) / 32 * 32;
    const int64_t per_pass = FLAT ? 1 : int64_t(kUnroll) << (8 - p.log2);
    for (int64_t row0 = blockIdx.y * per_pass; row0 < (FLAT ? 1 : p.rows); row0 += gridDim.y * per_pass) {
        Eight<TYPE> raw[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<FLAT, 8, kUnroll>(p, row0, i);
            raw[i].zero();
            if (at.in && (FLAT || at.col < p.cols)) raw[i].load(u + at.row * u_stride + at.col);
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<FLAT, 8, kUnroll>(p, row0, i);
            const int64_t to = code_at<FLAT>(p, at, pitch);
            F2 v[4];
            raw[i].get(v);
            if (uc.codes) put(uc, to, at.in, v, raw[i].top());
            if constexpr (KIND != kIdentity) {
                F2 f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = act<KIND>(v[k]);
                Eight<TYPE> out;
                out.set(f);
                if (a && at.in && (FLAT || at.col < p.cols)) out.store(a + at.row * a_stride + at.col);
                if (ac.codes) {         // of what the next layer reads: the rounded values
                    out.get(f);
                    put(ac, to, at.in, f, out.top());
                }
            }
        }
    }
}

template <int KIND, int TYPE, bool FLAT, bool FROM8>
__global__ void __launch_bounds__(kThreads)
novak_activation_backward_kernel(const typename Elem<TYPE>::T *da, int64_t da_stride, const typename Elem<TYPE>::T *u,
                                 int64_t u_stride, Codes uc, typename Elem<TYPE>::T *du, int64_t du_stride, Place p)
{
    const int64_t pitch = (p.cols + 31) / 32 * 32;
    const int64_t per_pass = FLAT ? 1 : int64_t(kUnroll) << (8 - p.log2);
    for (int64_t row0 = blockIdx.y * per_pass; row0 < (FLAT ? 1 : p.rows); row0 += gridDim.y * per_pass) {
        Eight<TYPE> raw[kUnroll], raw_u[FROM8 ? 1 : kUnroll];
        uint2 q[FROM8 ? kUnroll : 1];
        uint32_t e[FROM8 ? kUnroll : 1];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<FLAT, 8, kUnroll>(p, row0, i);
            if (!at.in || !(FLAT || at.col < p.cols)) continue;
            if constexpr (KIND != kIdentity) raw[i].load(da + at.row * da_stride + at.col);
            if constexpr (FROM8) {
                const int64_t from = code_at<FLAT>(p, at, pitch);
                q[i] = *reinterpret_cast<const uint2 *>(uc.codes + from);
                e[i] = uc.exps[from >> 5];
            } else {
                raw_u[i].load(u + at.row * u_stride + at.col);
            }
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<FLAT, 8, kUnroll>(p, row0, i);
            if (!at.in || !(FLAT || at.col < p.cols)) continue;
            F2 v[4];
            if constexpr (FROM8) dequantize8(q[i], e[i], v);
            else raw_u[i].get(v);
            if constexpr (KIND != kIdentity) {
                F2 g[4];
                raw[i].get(g);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = g[k] * act_slope<KIND>(v[k]);
            }
            Eight<TYPE> out;
            out.set(v);
            out.store(du + at.row * du_stride + at.col);
        }
    }
}

// Rows that are not aligned, or not a multiple of 8 long: neighbouring threads have
// neighbouring elements, a warp a block.
template <int KIND, int TYPE>
__global__ void __launch_bounds__(kThreads)
novak_activation_narrow_kernel(const typename Elem<TYPE>::T *u, int64_t u_stride, typename Elem<TYPE>::T *a,
                               int64_t a_stride, Codes uc, Codes ac, Place p)
{
    using T = typename Elem<TYPE>::T;
    const int64_t pitch = (p.cols + 31) / 32 * 32, per_pass = int64_t(kNarrowUnroll) << (8 - p.log2);
    auto put1 = [&](const Codes &c, const At &at, float v) {
        uint32_t exp;
        const uint8_t q = quantize1(v, exp);
        if (at.in) {
            const int64_t to = at.row * pitch + at.col;
            c.codes[to] = static_cast<int8_t>(q);
            if ((threadIdx.x & 31) == 0) c.exps[to >> 5] = static_cast<uint8_t>(exp);
        }
    };
    for (int64_t row0 = blockIdx.y * per_pass; row0 < p.rows; row0 += gridDim.y * per_pass) {
        T raw[kNarrowUnroll];
#pragma unroll
        for (int i = 0; i < kNarrowUnroll; ++i) {
            const At at = place<false, 1, kNarrowUnroll>(p, row0, i);
            raw[i] = at.in && at.col < p.cols ? u[at.row * u_stride + at.col] : from_float<T>(0.0f);
        }
#pragma unroll
        for (int i = 0; i < kNarrowUnroll; i += 2) {
            const At x = place<false, 1, kNarrowUnroll>(p, row0, i), y = place<false, 1, kNarrowUnroll>(p, row0, i + 1);
            const F2 v(to_float(raw[i]), to_float(raw[i + 1]));
            if (uc.codes) {
                put1(uc, x, v.lo());
                put1(uc, y, v.hi());
            }
            if constexpr (KIND != kIdentity) {
                const F2 f = act<KIND>(v);
                const T fx = from_float<T>(f.lo()), fy = from_float<T>(f.hi());
                if (a && x.in && x.col < p.cols) a[x.row * a_stride + x.col] = fx;
                if (a && y.in && y.col < p.cols) a[y.row * a_stride + y.col] = fy;
                if (ac.codes) {
                    put1(ac, x, to_float(fx));
                    put1(ac, y, to_float(fy));
                }
            }
        }
    }
}

template <int KIND, int TYPE, bool FROM8>
__global__ void __launch_bounds__(kThreads)
novak_activation_backward_narrow_kernel(const typename Elem<TYPE>::T *da, int64_t da_stride,
                                        const typename Elem<TYPE>::T *u, int64_t u_stride, Codes uc,
                                        typename Elem<TYPE>::T *du, int64_t du_stride, Place p)
{
    using T = typename Elem<TYPE>::T;
    const int64_t pitch = (p.cols + 31) / 32 * 32, per_pass = int64_t(kNarrowUnroll) << (8 - p.log2);
    for (int64_t row0 = blockIdx.y * per_pass; row0 < p.rows; row0 += gridDim.y * per_pass) {
        T raw[kNarrowUnroll], raw_u[FROM8 ? 1 : kNarrowUnroll];
        int8_t q[FROM8 ? kNarrowUnroll : 1];
        uint8_t e[FROM8 ? kNarrowUnroll : 1];
#pragma unroll
        for (int i = 0; i < kNarrowUnroll; ++i) {
            const At at = place<false, 1, kNarrowUnroll>(p, row0, i);
            const bool in = at.in && at.col < p.cols;
            if constexpr (KIND != kIdentity) raw[i] = in ? da[at.row * da_stride + at.col] : from_float<T>(0.0f);
            if constexpr (FROM8) {
                q[i] = in ? uc.codes[at.row * pitch + at.col] : 0;
                e[i] = in ? uc.exps[(at.row * pitch + at.col) >> 5] : 0;
            } else {
                raw_u[i] = in ? u[at.row * u_stride + at.col] : from_float<T>(0.0f);
            }
        }
#pragma unroll
        for (int i = 0; i < kNarrowUnroll; i += 2) {
            const At x = place<false, 1, kNarrowUnroll>(p, row0, i), y = place<false, 1, kNarrowUnroll>(p, row0, i + 1);
            F2 v;
            if constexpr (FROM8)
                v = F2(static_cast<float>(q[i]) * scale_of(e[i]), static_cast<float>(q[i + 1]) * scale_of(e[i + 1]));
            else
                v = F2(to_float(raw_u[i]), to_float(raw_u[i + 1]));
            if constexpr (KIND != kIdentity) v = F2(to_float(raw[i]), to_float(raw[i + 1])) * act_slope<KIND>(v);
            if (x.in && x.col < p.cols) du[x.row * du_stride + x.col] = from_float<T>(v.lo());
            if (y.in && y.col < p.cols) du[y.row * du_stride + y.col] = from_float<T>(v.hi());
        }
    }
}

// The grid for `groups` per row of which 256 threads take 2^log2 per row.
dim3 spread(Place &p, int64_t per_row, int unroll)
{
    p.groups = per_row;
    p.log2 = 5;             // a warp is in one row
    while (p.log2 < 8 && (int64_t(1) << p.log2) < per_row) ++p.log2;
    const int64_t x = (per_row + (int64_t(1) << p.log2) - 1) >> p.log2, per_pass = int64_t(unroll) << (8 - p.log2);
    return dim3(static_cast<unsigned>(x), static_cast<unsigned>(std::min<int64_t>((p.rows + per_pass - 1) / per_pass, 65535)));
}

// One run of elements: every matrix that is there has rows of a multiple of 32 with no
// gaps.
bool is_flat(const Mat &m, int64_t rows, int64_t cols) { return !m.ptr || rows <= 1 || m.stride == cols; }

dim3 spread_flat(Place &p)
{
    p.groups = p.rows * p.cols / 8;
    return dim3(static_cast<unsigned>((p.groups + kThreads * kUnroll - 1) / (kThreads * kUnroll)));
}

template <int KIND, int TYPE>
cudaError_t forward(Mat u, Mat a, Codes uc, Codes ac, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    Place p{rows, cols, 0, 0};
    const T *up = static_cast<const T *>(u.ptr);
    T *ap = static_cast<T *>(a.ptr);
    if (cols % 8 || !wide(u, TYPE, rows) || (a.ptr && !wide(a, TYPE, rows))) {
        const dim3 grid = spread(p, act_pitch(cols), kNarrowUnroll);
        novak_activation_narrow_kernel<KIND, TYPE><<<grid, kThreads, 0, stream>>>(up, u.stride, ap, a.stride, uc, ac, p);
    } else if (cols % 32 == 0 && is_flat(u, rows, cols) && is_flat(a, rows, cols) && rows * cols < (int64_t(1) << 42)) {
        const dim3 grid = spread_flat(p);
        novak_activation_kernel<KIND, TYPE, true><<<grid, kThreads, 0, stream>>>(up, u.stride, ap, a.stride, uc, ac, p);
    } else {
        const dim3 grid = spread(p, act_pitch(cols) / 8, kUnroll);
        novak_activation_kernel<KIND, TYPE, false><<<grid, kThreads, 0, stream>>>(up, u.stride, ap, a.stride, uc, ac, p);
    }
    return cudaGetLastError();
}

template <int KIND, int TYPE, bool FROM8>
cudaError_t backward(Mat da, Mat u, Codes uc, Mat du, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    Place p{rows, cols, 0, 0};
    const T *dap = static_cast<const T *>(da.ptr), *up = static_cast<const T *>(u.ptr);
    T *dup = static_cast<T *>(du.ptr);
    if (cols % 8 || (da.ptr && !wide(da, TYPE, rows)) || (u.ptr && !wide(u, TYPE, rows)) || !wide(du, TYPE, rows)) {
        const dim3 grid = spread(p, act_pitch(cols), kNarrowUnroll);
        novak_activation_backward_narrow_kernel<KIND, TYPE, FROM8><<<grid, kThreads, 0, stream>>>(dap, da.stride, up, u.stride, uc, dup, du.stride, p);
    } else if (cols % 32 == 0 && is_flat(da, rows, cols) && is_flat(u, rows, cols) && is_flat(du, rows, cols) &&
               rows * cols < (int64_t(1) << 42)) {
        const dim3 grid = spread_flat(p);
        novak_activation_backward_kernel<KIND, TYPE, true, FROM8><<<grid, kThreads, 0, stream>>>(dap, da.stride, up, u.stride, uc, dup, du.stride, p);
    } else {
        const dim3 grid = spread(p, act_pitch(cols) / 8, kUnroll);
        novak_activation_backward_kernel<KIND, TYPE, false, FROM8><<<grid, kThreads, 0, stream>>>(dap, da.stride, up, u.stride, uc, dup, du.stride, p);
    }
    return cudaGetLastError();
}

template <int KIND>
cudaError_t backward_kind(Mat da, Mat u, int type, Codes uc, Mat du, int64_t rows, int64_t cols, cudaStream_t stream)
{
    if (uc.codes)
        return type == NOVAK_TYPE_F32 ? backward<KIND, NOVAK_TYPE_F32, true>(da, u, uc, du, rows, cols, stream)
                                      : backward<KIND, NOVAK_TYPE_BF16, true>(da, u, uc, du, rows, cols, stream);
    if constexpr (KIND != kIdentity)
        return type == NOVAK_TYPE_F32 ? backward<KIND, NOVAK_TYPE_F32, false>(da, u, uc, du, rows, cols, stream)
                                      : backward<KIND, NOVAK_TYPE_BF16, false>(da, u, uc, du, rows, cols, stream);
    return cudaErrorInvalidValue;
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
    switch (kind) {
        case NOVAK_ACT_GELU: return backward_kind<NOVAK_ACT_GELU>(da, u, type, uc, du, rows, cols, stream);
        case NOVAK_ACT_GELU_TANH: return backward_kind<NOVAK_ACT_GELU_TANH>(da, u, type, uc, du, rows, cols, stream);
        case NOVAK_ACT_SILU: return backward_kind<NOVAK_ACT_SILU>(da, u, type, uc, du, rows, cols, stream);
        case kIdentity: return backward_kind<kIdentity>(da, u, type, uc, du, rows, cols, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace novak
