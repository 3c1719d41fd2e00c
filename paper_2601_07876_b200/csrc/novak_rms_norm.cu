// Root-mean-square norm with the residual's addition in front, forward and backward.
//     h = x + r, rounded to the stream's type, rstd = 1/sqrt(sum(h^2)/C + eps), xhat = h rstd,
//     y = xhat w;
//     g = dy w, dx = dh + rstd (g - xhat sum(g xhat)/C), dw = sum over rows of dy xhat.
// What is normalised is h as it is stored, so that the backward pass, which may form xhat from
// it, sees what the forward pass saw.  Rows are spread as the layer norm's are: read once,
// held in registers, the next one on its way; one sum over the row's threads where the layer
// norm has two.  Bound by HBM where there are rows enough: 12608 x 768 bf16 with a residual, the 8-bit
// form left and unpacked, 21.4 us (18.0 at the copy rate); back from that form with a stream's gradient 19.6
// (10.5: few rows per warp, and a second kernel of 5 us for dw's sums); back from h, 4099 x 4096 fp32, 53.5 (41.6).
#include <algorithm>

#include "novak_norm.cuh"

namespace novak {
namespace {

// 1 / sqrt(sum / cols + eps), each operation correctly rounded: codes of the 8-bit form are whole numbers, and every ulp of
// rstd's turns some of them over.  Of 12608 rows of 768 bf16 some 2470 are then not the nearest to the exact one (with
// the approximate root, 2 ulp, and a product with 1 / cols 3490), and the call takes as long.
__device__ __forceinline__ float reciprocal_root(float sum, int64_t cols, float eps)
{
    return __frsqrt_rn(__fadd_rn(__fdiv_rn(sum, static_cast<float>(cols)), eps));
}

// ---- rows in registers -------------------------------------------------------------------
template <int TYPE, int G, int NV, bool ALIGNED, bool RESIDUAL>
__global__ void __launch_bounds__(32 * forward_warps<G, NV>()) novak_rms_norm_kernel(RmsArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[G == 32 ? 1 : 2 * 32];
    __shared__ __align__(16) float held[G == 32 ? NV * 256 : 4];
    int turn = 0;
    const int t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0;
    constexpr int kSubs = G == 32 ? forward_warps<G, NV>() : 1;
    const int cols = static_cast<int>(a.cols), pitch = (cols + 31) / 32 * 32;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kSubs;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kSubs + sub;
    const T *x = static_cast<const T *>(a.x.ptr) + row * a.x.stride + t * 8;
    const T *r = static_cast<const T *>(a.residual.ptr) + row * a.residual.stride + t * 8;
    T *h = static_cast<T *>(a.h.ptr) + row * a.h.stride + t * 8;
    T *y = static_cast<T *>(a.y.ptr) + row * a.y.stride + t * 8;
    const void *x_end = end_of(static_cast<const T *>(a.x.ptr), a.x.stride, a.rows, cols);
    const void *r_end = end_of(static_cast<const T *>(a.residual.ptr), a.residual.stride, a.rows, cols);
    int n[NV];                  // elements of a group inside the row
    Fetch<TYPE, ALIGNED> raw[NV], raw_r[RESIDUAL ? NV : 1];
    start();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        n[i] = max(min(cols - (i * G + t) * 8, 8), 0);
        raw[i].zero();
        if (row < a.rows) raw[i].load(x + i * G * 8, n[i], a.x.ptr, x_end);
        if constexpr (RESIDUAL) {
            raw_r[i].zero();
            if (row < a.rows) raw_r[i].load(r + i * G * 8, n[i], a.residual.ptr, r_end);
        }
    }
    Held<G, NV> weight;
    weight.load(a.weight, a.param_type, cols, held);
    if constexpr (G == 32) __syncthreads();
    for (; row < a.rows; row += step, y += step * a.y.stride) {
        F2 v[NV][4], sum(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].eight().get(v[i]);
            if constexpr (RESIDUAL) {
                F2 b[4];
                raw_r[i].eight().get(b);
                Eight<TYPE> out;
#pragma unroll
                for (int k = 0; k < 4; ++k) b[k] = v[i][k] + b[k];
                out.set(b);
                store_eight<ALIGNED>(h + i * G * 8, out, n[i]);
                out.get(v[i]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = fma2(v[i][k], v[i][k], sum);
        }
        x += step * a.x.stride;
        if constexpr (RESIDUAL) {
            r += step * a.residual.stride;
            h += step * a.h.stride;
        }
        if (row + step < a.rows)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                raw[i].load(x + i * G * 8, n[i], a.x.ptr, x_end);
                if constexpr (RESIDUAL) raw_r[i].load(r + i * G * 8, n[i], a.residual.ptr, r_end);
            }
        float s[1] = {sum.lo() + sum.hi()};
        row_sums<G, 1>(s, scratch, turn);
        const float rstd = reciprocal_root(s[0], cols, a.eps);
        if (t == 0 && a.rstd) a.rstd[row] = rstd;
        const F2 r2(rstd);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            F2 o[4], w[4];
            weight.get(i, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = v[i][k] * r2;
                o[k] = v[i][k] * w[k];
            }
            Eight<TYPE> out;
            out.set(o);
            store_eight<ALIGNED>(y + i * G * 8, out, n[i]);
            if (a.codes.codes) put_codes(a.codes, row, pitch, (i * G + t) * 8, v[i]);
        }
    }
}

// A thread's columns of dw are added up in registers over the CTA's rows and go to
// work[CTA][cols], which the finish kernel adds up in order.
template <int TYPE, int G, int NV, bool ALIGNED, bool FROM8>
__global__ void __launch_bounds__(32 * backward_warps<G, NV>(), G == 256 ? 2 : 1)
novak_rms_norm_back_kernel(RmsBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[G == 32 ? 1 : 2 * 32];
    extern __shared__ __align__(16) float held[];       // warps: the weight, then the warps' column sums
    int turn = 0;
    const int t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0;
    constexpr int kWarps = backward_warps<G, NV>(), kSubs = G == 32 ? kWarps : 1;
    const int cols = static_cast<int>(a.cols), pitch = (cols + 31) / 32 * 32;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kSubs;
    const float inv_cols = 1.0f / static_cast<float>(cols);
    int64_t row = static_cast<int64_t>(blockIdx.x) * kSubs + sub;
    const bool stream = a.dh.ptr != nullptr;
    const T *dy = static_cast<const T *>(a.dy.ptr) + row * a.dy.stride + t * 8;
    const T *dh = static_cast<const T *>(a.dh.ptr) + row * a.dh.stride + t * 8;
    const T *h = static_cast<const T *>(a.h.ptr) + row * a.h.stride + t * 8;
    const int8_t *codes = a.codes.codes + row * pitch + t * 8;
    const uint8_t *exps = a.codes.exps + row * (pitch / 32) + t / 4;
    T *dx = static_cast<T *>(a.dx.ptr) + row * a.dx.stride + t * 8;
    const void *dy_end = end_of(static_cast<const T *>(a.dy.ptr), a.dy.stride, a.rows, cols);
    const void *dh_end = end_of(static_cast<const T *>(a.dh.ptr), a.dh.stride, a.rows, cols);
    const void *h_end = end_of(static_cast<const T *>(a.h.ptr), a.h.stride, a.rows, cols);
    int n[NV];
    Fetch<TYPE, ALIGNED> raw[NV], raw_d[NV], raw_h[FROM8 ? 1 : NV];
    uint2 q[FROM8 ? NV : 1];
    uint32_t e[FROM8 ? NV : 1];
    float rstd = 0.0f;
    auto fetch = [&](int64_t at) {
        if (at >= a.rows) return;
        rstd = a.rstd[at];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].load(dy + i * G * 8, n[i], a.dy.ptr, dy_end);
            if (stream) raw_d[i].load(dh + i * G * 8, n[i], a.dh.ptr, dh_end);
            if constexpr (FROM8) {
                if (n[i] > 0) {
                    q[i] = *reinterpret_cast<const uint2 *>(codes + i * G * 8);
                    e[i] = exps[i * G / 4];
                }
            } else {
                raw_h[i].load(h + i * G * 8, n[i], a.h.ptr, h_end);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        n[i] = max(min(cols - (i * G + t) * 8, 8), 0);
        raw[i].zero();
        raw_d[i].zero();
        if constexpr (FROM8) {
            q[i] = make_uint2(0, 0);
            e[i] = 0;
        } else {
            raw_h[i].zero();
        }
    }
    start();
    fetch(row);
    Held<G, NV> weight;
    weight.load(a.weight, a.param_type, cols, held);
    if constexpr (G == 32) __syncthreads();
    F2 dw[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[i][k] = F2(0.0f);
    for (; row < a.rows; row += step, dx += step * a.dx.stride) {
        // (beyond the row dy, codes or h, and the weight are zeros: xhat is finite there)
        F2 g[NV][4], xh[NV][4], d[NV][4], s0(0.0f);
        const F2 r2(rstd);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].eight().get(g[i]);
            raw_d[i].eight().get(d[i]);
            if constexpr (FROM8) dequantize8(q[i], e[i], xh[i]);
            else raw_h[i].eight().get(xh[i]);
            F2 w[4];
            weight.get(i, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!FROM8) xh[i][k] = xh[i][k] * r2;
                dw[i][k] = fma2(g[i][k], xh[i][k], dw[i][k]);
                g[i][k] = g[i][k] * w[k];
                s0 = fma2(g[i][k], xh[i][k], s0);
            }
        }
        const float r = rstd;
        dy += step * a.dy.stride;
        if (stream) dh += step * a.dh.stride;
        if constexpr (FROM8) {
            codes += step * pitch;
            exps += step * (pitch / 32);
        } else {
            h += step * a.h.stride;
        }
        fetch(row + step);
        float s[1] = {s0.lo() + s0.hi()};
        row_sums<G, 1>(s, scratch, turn);
        const F2 a1(-s[0] * inv_cols * r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) g[i][k] = fma2(g[i][k], r2, fma2(xh[i][k], a1, d[i][k]));
            Eight<TYPE> out;
            out.set(g[i]);
            store_eight<ALIGNED>(dx + i * G * 8, out, n[i]);
        }
    }
    if (!a.dweight) return;
    float *out = a.work + static_cast<int64_t>(blockIdx.x) * cols;
    if constexpr (G == 32) {
        float *part = held + NV * 256;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<float4 *>(part + sub * NV * 256 + Held<G, NV>::at(i, 4 * k, t)) =
                    make_float4(dw[i][2 * k].lo(), dw[i][2 * k].hi(), dw[i][2 * k + 1].lo(), dw[i][2 * k + 1].hi());
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const int at = Held<G, NV>::at(c / 256, c % 8, c / 8 % 32);
            float sum = 0.0f;
#pragma unroll
            for (int p = 0; p < kWarps; ++p) sum += part[p * NV * 256 + at];
            out[c] = sum;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int col = (i * G + t) * 8 + 2 * k;
                if (2 * k < n[i]) out[col] = dw[i][k].lo();
                if (2 * k + 1 < n[i]) out[col + 1] = dw[i][k].hi();
            }
    }
}

// ---- rows too long for registers ---------------------------------------------------------
// One CTA per row, any length: the row is read twice, from L2 the second time.  A thread
// reads back from h what it wrote there itself.
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_rms_norm_long_kernel(RmsArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[33];
    start();
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const bool add = a.residual.ptr != nullptr;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x.ptr) + row * a.x.stride;
        const T *r = static_cast<const T *>(a.residual.ptr) + row * a.residual.stride;
        T *h = static_cast<T *>(a.h.ptr) + row * a.h.stride, *y = static_cast<T *>(a.y.ptr) + row * a.y.stride;
        float sum = 0.0f, v[8];
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(x, c, a.cols, v);
            if (add) {
                float b[8];
                load8<WIDE>(r, c, a.cols, b);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = to_float(T(v[k] + b[k]));
                store8<WIDE>(h, c, a.cols, v);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
        }
        const float rstd = reciprocal_root(block_sum(sum, scratch), a.cols, a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
        // (the pitch is a multiple of 32: a quad is inside it, or outside, as a whole)
        for (int64_t c0 = 0; c0 < pitch; c0 += kThreads * 8) {
            const int64_t c = c0 + threadIdx.x * 8;
            load8<WIDE>(add ? h : x, c, a.cols, v);
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] *= c + k < a.cols ? rstd : 0.0f;
                o[k] = c + k < a.cols ? v[k] * param_at(a.weight, a.param_type, c + k) : 0.0f;
            }
            store8<WIDE>(y, c, a.cols, o);
            if (a.codes.codes) {
                F2 p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) p[k] = F2(v[2 * k], v[2 * k + 1]);
                put_codes(a.codes, row, pitch, c, p);
            }
        }
    }
}

// xhat of eight elements, from the 8-bit form or from h.
template <int TYPE, bool WIDE>
__device__ __forceinline__ void rms_xhat8(const RmsBackArgs &a, int64_t row, int64_t c, int64_t pitch, float rstd,
                                          float (&v)[8])
{
    if (a.codes.codes) {
        dequantize8(*reinterpret_cast<const uint2 *>(a.codes.codes + row * pitch + c),
                    a.codes.exps[(row * pitch + c) >> 5], v);
    } else {
        using T = typename Elem<TYPE>::T;
        load8<WIDE>(static_cast<const T *>(a.h.ptr) + row * a.h.stride, c, a.cols, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < a.cols ? v[k] * rstd : 0.0f;
    }
}

template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_rms_norm_back_long_kernel(RmsBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[33];
    start();
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const float inv_cols = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dy.ptr) + row * a.dy.stride;
        const T *dh = static_cast<const T *>(a.dh.ptr) + row * a.dh.stride;
        T *dx = static_cast<T *>(a.dx.ptr) + row * a.dx.stride;
        const float rstd = a.rstd[row];
        float s = 0.0f, g[8], xh[8], d[8] = {};
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(dy, c, a.cols, g);
            rms_xhat8<TYPE, WIDE>(a, row, c, pitch, rstd, xh);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < a.cols) s = fmaf(g[k] * param_at(a.weight, a.param_type, c + k), xh[k], s);
        }
        s = block_sum(s, scratch) * inv_cols;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8<WIDE>(dy, c, a.cols, g);
            rms_xhat8<TYPE, WIDE>(a, row, c, pitch, rstd, xh);
            if (a.dh.ptr) load8<WIDE>(dh, c, a.cols, d);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < a.cols)
                    g[k] = fmaf(rstd, fmaf(-xh[k], s, g[k] * param_at(a.weight, a.param_type, c + k)), d[k]);
            store8<WIDE>(dx, c, a.cols, g);
        }
    }
}

// Column sums of dy xhat over kSplitRows rows at a time: 32 columns per CTA,
// partial[split][cols].
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_rms_norm_columns_kernel(RmsBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float part[kThreads / 4][kColsPerCta + 1];
    start();
    const int64_t pitch = (a.cols + 31) / 32 * 32;
    const int quad = threadIdx.x & 3, lane = threadIdx.x >> 2;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kColsPerCta + quad * 8;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kSplitRows;
    const int64_t row1 = min(row0 + kSplitRows, a.rows);
    float dw[8] = {}, g[8], xh[8];
    for (int64_t row = row0 + lane; row < row1; row += kThreads / 4) {
        load8<WIDE>(static_cast<const T *>(a.dy.ptr) + row * a.dy.stride, c, a.cols, g);
        rms_xhat8<TYPE, WIDE>(a, row, c, pitch, a.rstd[row], xh);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < a.cols) dw[k] = fmaf(g[k], xh[k], dw[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) part[lane][quad * 8 + k] = dw[k];
    __syncthreads();
    if (threadIdx.x < kColsPerCta) {
        float s = 0.0f;
        for (int i = 0; i < kThreads / 4; ++i) s += part[i][threadIdx.x];
        const int64_t out = static_cast<int64_t>(blockIdx.x) * kColsPerCta + threadIdx.x;
        if (out < a.cols) a.work[static_cast<int64_t>(blockIdx.y) * a.cols + out] = s;
    }
}

// CTAs of the backward pass, each of which leaves one partial sum per column.
int64_t rms_back_ctas(const Spread &s, int64_t rows)
{
    const int per_sm = s.g == 32 || s.g == 512 ? 1 : s.g == 128 ? 4 : 2;
    return std::min<int64_t>(rows, kSms * per_sm);
}

// CTAs per SM of the forward pass: what registers leave room for.
constexpr int rms_forward_ctas(int type, int g, int nv)
{
    return g == 32 ? 4 : g == 256 ? (nv == 1 ? 4 : type == NOVAK_TYPE_F32 ? 2 : 3) : 1024 / g / nv;
}

template <int TYPE, bool RESIDUAL> cudaError_t rms_forward(const RmsArgs &a, const Spread &s, bool aligned, cudaStream_t stream)
{
#define NOVAK_CASE(G, NV, ALIGNED)                                                                                        \
    if (s.g == G && s.nv == NV && aligned == ALIGNED) {                                                                   \
        constexpr int warps = forward_warps<G, NV>(), rows = G == 32 ? warps : 1;                                         \
        const int64_t grid = std::min<int64_t>((a.rows + rows - 1) / rows, kSms * rms_forward_ctas(TYPE, G, NV));         \
        return launch(novak_rms_norm_kernel<TYPE, G, NV, ALIGNED, RESIDUAL>, dim3(static_cast<unsigned>(grid)), 32 * warps, \
                      0, stream, a);                                                                                      \
    }
    NOVAK_SPREADS(NOVAK_CASE)
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

template <int TYPE, bool FROM8>
cudaError_t rms_backward(const RmsBackArgs &a, const Spread &s, bool aligned, int64_t grid, cudaStream_t stream)
{
#define NOVAK_CASE(G, NV, ALIGNED)                                                                                    \
    if (s.g == G && s.nv == NV && aligned == ALIGNED) {                                                               \
        constexpr int warps = backward_warps<G, NV>(), smem = G == 32 ? (1 + warps) * NV * 256 * 4 : 0;               \
        static_assert(smem <= 40 * 1024, "48 KB without asking, less the kernel's own");                              \
        return launch(novak_rms_norm_back_kernel<TYPE, G, NV, ALIGNED, FROM8>, dim3(static_cast<unsigned>(grid)),     \
                      32 * warps, smem, stream, a);                                                                   \
    }
    NOVAK_SPREADS(NOVAK_CASE)
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

template <int TYPE> cudaError_t rms_forward_of(const RmsArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.x, a.type, a.rows) && wide(a.y, a.type, a.rows) &&
                   (!a.residual.ptr || (wide(a.residual, a.type, a.rows) && wide(a.h, a.type, a.rows)));
    const bool aligned = w && a.cols % 8 == 0;
    Spread s;
    if (aligned ? spread_for(kAlignedRows, a.cols, s) : spread_for(kAnyRows, a.cols, s))
        return a.residual.ptr ? rms_forward<TYPE, true>(a, s, aligned, stream) : rms_forward<TYPE, false>(a, s, aligned, stream);
    const int64_t grid = std::min<int64_t>(a.rows, kSms * 8);
    return launch(w ? novak_rms_norm_long_kernel<TYPE, true> : novak_rms_norm_long_kernel<TYPE, false>,
                  dim3(static_cast<unsigned>(grid)), kThreads, 0, stream, a);
}

template <int TYPE> cudaError_t rms_backward_of(const RmsBackArgs &a, int64_t &splits, cudaStream_t stream)
{
    const bool w = wide(a.dy, a.type, a.rows) && wide(a.dx, a.type, a.rows) && (!a.h.ptr || wide(a.h, a.type, a.rows)) &&
                   (!a.dh.ptr || wide(a.dh, a.type, a.rows));
    const bool aligned = w && a.cols % 8 == 0;
    Spread s;
    if (aligned ? spread_for(kAlignedRows, a.cols, s) : spread_for(kAnyRows, a.cols, s)) {
        splits = rms_back_ctas(s, a.rows);
        return a.codes.codes ? rms_backward<TYPE, true>(a, s, aligned, splits, stream)
                             : rms_backward<TYPE, false>(a, s, aligned, splits, stream);
    }
    splits = (a.rows + kSplitRows - 1) / kSplitRows;
    if (a.dweight) {            // first: dx may be written over dy
        // (splits fit the grid's second dimension: it holds up to 65535 of them)
        for (int64_t at = 0; at < splits; at += 65535) {
            RmsBackArgs part = a;
            const int64_t row = at * kSplitRows;
            using T = typename Elem<TYPE>::T;
            part.dy.ptr = static_cast<T *>(a.dy.ptr) + row * a.dy.stride;
            if (a.h.ptr) part.h.ptr = static_cast<T *>(a.h.ptr) + row * a.h.stride;
            if (a.codes.codes) part.codes = Codes{a.codes.codes + row * act_pitch(a.cols), a.codes.exps + row * (act_pitch(a.cols) / kActBlock)};
            part.rstd = a.rstd + row;
            part.work = a.work + at * a.cols;
            part.rows = a.rows - row;
            const dim3 grid(static_cast<unsigned>((a.cols + kColsPerCta - 1) / kColsPerCta),
                            static_cast<unsigned>(std::min<int64_t>(splits - at, 65535)));
            const cudaError_t e = launch(w ? novak_rms_norm_columns_kernel<TYPE, true> : novak_rms_norm_columns_kernel<TYPE, false>,
                                         grid, kThreads, 0, stream, part);
            if (e != cudaSuccess) return e;
        }
    }
    return launch(w ? novak_rms_norm_back_long_kernel<TYPE, true> : novak_rms_norm_back_long_kernel<TYPE, false>,
                  dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kSms * 8))), kThreads, 0, stream, a);
}

}  // namespace

cudaError_t launch_rms_norm(const RmsArgs &a, cudaStream_t stream)
{
    return a.type == NOVAK_TYPE_F32 ? rms_forward_of<NOVAK_TYPE_F32>(a, stream) : rms_forward_of<NOVAK_TYPE_BF16>(a, stream);
}

// Enough for either way of the backward pass: which one it is depends on alignment.
size_t rms_norm_backward_bytes(int64_t rows, int64_t cols)
{
    int64_t splits = (rows + kSplitRows - 1) / kSplitRows;
    Spread s;
    if (spread_for(kAnyRows, cols, s)) splits = std::max(splits, rms_back_ctas(s, rows));
    if (spread_for(kAlignedRows, cols, s)) splits = std::max(splits, rms_back_ctas(s, rows));
    return static_cast<size_t>(splits * cols) * sizeof(float);
}

cudaError_t launch_rms_norm_backward(const RmsBackArgs &a, cudaStream_t stream)
{
    int64_t splits = 0;
    if (a.rows > 0) {
        const cudaError_t e = a.type == NOVAK_TYPE_F32 ? rms_backward_of<NOVAK_TYPE_F32>(a, splits, stream)
                                                       : rms_backward_of<NOVAK_TYPE_BF16>(a, splits, stream);
        if (e != cudaSuccess) return e;
    }
    if (!a.dweight) return cudaSuccess;
    return launch(novak_layer_norm_finish_kernel, dim3(static_cast<unsigned>((a.cols + 31) / 32)), kFinishThreads, 0, stream,
                  static_cast<const float *>(a.work), splits, a.cols, 1, a.dweight, static_cast<void *>(nullptr), a.grad_type);
}

}  // namespace novak
