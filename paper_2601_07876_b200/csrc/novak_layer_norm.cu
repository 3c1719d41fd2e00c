// Layer norm, forward and backward.
//     mean = sum(x)/C, rstd = 1/sqrt(sum((x - mean)^2)/C + eps), xhat = (x - mean) rstd,
//     y = xhat w + b;
//     g = dy w, dx = rstd (g - sum(g)/C - xhat sum(g xhat)/C),
//     dw = sum over rows of dy xhat, db = sum over rows of dy.
// A row is read once and stays in registers: the deviations are summed after the mean
// is known.  A thread has eight neighbouring elements at a time and computes on pairs.
// Rows that are not 16-byte aligned, or not a multiple of 8 elements long, are read and
// written as the aligned pieces that hold them.  Rows too long for registers (more than
// 8192 elements) have kernels of their own.
//
// Up to 1024 elements a row is a warp's and needs no barrier; wider ones are 256 or 512
// threads'.  What bounds them is not bytes but what a row has to wait for, its load, two
// sums over its threads one after the other, at the occupancy that its registers leave:
//   forward with the 8-bit form left: 12608 x 768 bf16 12.6 us (3.9 TB/s), 8000 x 4096 bf16 32.2
//   (5.1), 4099 x 4096 fp32 28.5 (5.3);
//   backward: 12608 x 768 bf16 11.8 us (4.1 TB/s; 18.4 with other inputs each time), 8000 x 4096
//   bf16 50 (3.2), 4099 x 4096 fp32 from x 41.4 (4.9), 5 to 6 us of each for the last sums of
//   dw and db (single calls, one after the other on the same inputs).  (4096 columns: 282 instructions per warp and row at 40 % of the issue
//   slots; stalls on loads, shuffles, barriers and the load queue in like parts.)
//   Not aligned: 12608 x 771 bf16 25.4 and 27.1 us.  Long: 2000 x 20000 bf16 122 and 186.
//   One row of 768: 3.6 us.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;
constexpr int kSplitRows = 128;      // rows per partial sum of a column (long rows)
constexpr int kColsPerCta = 32;
constexpr int kSms = 148;

// Puts the 8-bit form of a thread's eight elements at `col` of `row` away; every thread
// of the warp has to be here, with zeros beyond the row's elements.
__device__ __forceinline__ void put_codes(const Codes &c, int64_t row, int64_t pitch, int64_t col, const F2 (&v)[4])
{
    uint32_t exp;
    const uint2 q = quantize8(v, top_of(v), exp);
    if (col < pitch) {
        const int64_t at = row * pitch + col;
        *reinterpret_cast<uint2 *>(c.codes + at) = q;
        if ((threadIdx.x & 3) == 0) c.exps[at >> 5] = static_cast<uint8_t>(exp);
    }
}

// Sums of N values over the G threads of a row, in every thread.  `scratch` (G > 32):
// two halves of 32 N floats, used in turn, so that one barrier per call is enough.
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float *scratch, int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = warp_sum(x[i]);
    if constexpr (G > 32) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        float *s = scratch + turn * 32 * N;
        turn ^= 1;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i * 32 + warp] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = lane < G / 32 ? s[i * 32 + lane] : 0.0f;
#pragma unroll
            for (int d = G / 64; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
            x[i] = __shfl_sync(0xffffffffu, t, 0);
        }
    }
}

// Warps per CTA: where a row is a warp's (G = 32), what the registers of a row of NV
// groups of 8 elements per lane leave room for (backward of 12608 x 768: 12 warps, which
// spill, 14.4 us in bf16 and 22.6 in fp32; 8 warps 13.0 and 17.3; two rows ahead of 8
// warps 12.6 and 17.3, of 12 warps 20 and 36).
template <int G, int NV> __host__ __device__ constexpr int forward_warps() { return G == 32 ? 8 : G / 32; }
template <int G, int NV> __host__ __device__ constexpr int backward_warps()
{
    return G == 32 ? (NV <= 2 ? 16 : 8) : G / 32;
}

// A thread's columns of a vector that every row needs.  Where a row is a warp's, the
// warps of a CTA share one copy in shared memory, in the order in which lanes read
// it; elsewhere it stays in registers.
template <int G, int NV> struct Held {
    F2 r[NV][4];
    __device__ __forceinline__ void load(const void *p, int type, int cols, float *)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * G + static_cast<int>(threadIdx.x)) * 8;
#pragma unroll
            for (int k = 0; k < 4; ++k)         // (the row's end may cut a group: nothing is read beyond it)
                r[i][k] = F2(p && col + 2 * k < cols ? param_at(p, type, col + 2 * k) : 0.0f,
                             p && col + 2 * k + 1 < cols ? param_at(p, type, col + 2 * k + 1) : 0.0f);
        }
    }
    __device__ __forceinline__ void get(int i, F2 (&v)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = r[i][k];
    }
};
template <int NV> struct Held<32, NV> {
    const float *s;
    // element k of lane t's i-th group: four to a lane
    static __device__ __forceinline__ int at(int i, int k, int t) { return ((i * 2 + k / 4) * 32 + t) * 4 + k % 4; }
    __device__ __forceinline__ void load(const void *p, int type, int cols, float *smem)
    {
        for (int c = threadIdx.x; c < NV * 256; c += blockDim.x)
            smem[at(c / 256, c % 8, c / 8 % 32)] = p && c < cols ? param_at(p, type, c) : 0.0f;
        s = smem;
    }
    __device__ __forceinline__ void get(int i, F2 (&v)[4]) const
    {
        const int t = threadIdx.x & 31;
        const float4 a = *reinterpret_cast<const float4 *>(s + at(i, 0, t)), b = *reinterpret_cast<const float4 *>(s + at(i, 4, t));
        v[0] = F2(a.x, a.y);
        v[1] = F2(a.z, a.w);
        v[2] = F2(b.x, b.y);
        v[3] = F2(b.z, b.w);
    }
};

// ---- rows in registers -------------------------------------------------------------------
// G threads per row, NV groups of 8 each; the next row is on its way while this one is
// worked on.
template <int TYPE, int G, int NV, bool ALIGNED>
__global__ void __launch_bounds__(32 * forward_warps<G, NV>()) novak_layer_norm_kernel(NormArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[G == 32 ? 1 : 2 * 32];
    __shared__ __align__(16) float held[G == 32 ? 2 * NV * 256 : 4];
    int turn = 0;
    const int t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0;
    constexpr int kSubs = G == 32 ? forward_warps<G, NV>() : 1;
    const int cols = static_cast<int>(a.cols), pitch = (cols + 31) / 32 * 32;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kSubs;
    const float inv_cols = 1.0f / static_cast<float>(cols);
    int64_t row = static_cast<int64_t>(blockIdx.x) * kSubs + sub;
    const T *x = static_cast<const T *>(a.x.ptr) + row * a.x.stride + t * 8;
    T *y = static_cast<T *>(a.y.ptr) + row * a.y.stride + t * 8;
    const void *end = end_of(static_cast<const T *>(a.x.ptr), a.x.stride, a.rows, cols);
    int n[NV];                  // elements of a group inside the row
    Fetch<TYPE, ALIGNED> raw[NV];
    start();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        n[i] = max(min(cols - (i * G + t) * 8, 8), 0);
        raw[i].zero();
        if (row < a.rows) raw[i].load(x + i * G * 8, n[i], a.x.ptr, end);
    }
    Held<G, NV> weight, bias;
    weight.load(a.weight, a.param_type, cols, held);
    bias.load(a.bias, a.param_type, cols, held + (G == 32 ? NV * 256 : 0));
    if constexpr (G == 32) __syncthreads();
    for (; row < a.rows; row += step, y += step * a.y.stride) {
        F2 v[NV][4], sum(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].eight().get(v[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = sum + v[i][k];
        }
        x += step * a.x.stride;
        if (row + step < a.rows)
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[i].load(x + i * G * 8, n[i], a.x.ptr, end);
        float s[1] = {sum.lo() + sum.hi()};
        row_sums<G, 1>(s, scratch, turn);
        const float mean = s[0] * inv_cols;
        sum = F2(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const F2 m(n[i] > 0 ? -mean : 0.0f);        // zeros stay zeros beyond the row
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = v[i][k] + (ALIGNED ? m : F2(2 * k < n[i] ? -mean : 0.0f, 2 * k + 1 < n[i] ? -mean : 0.0f));
                sum = fma2(v[i][k], v[i][k], sum);
            }
        }
        s[0] = sum.lo() + sum.hi();
        row_sums<G, 1>(s, scratch, turn);
        // (to 2 ulp.  A root and a division, as for long rows, cost 0.4 us of 12 and leave as many of
        // xhat's codes on the other side of halfway: of 58 million 72, this 73.  By one fp32 operation
        // of torch's after another it is as many: of 390 million 527, this 522.  A step of Newton's
        // on it and codes from products that are not rounded: 336, for 0.6 us of 12 and 9 of 17
        // at 4096 columns)
        const float rstd = rsqrtf(fmaf(s[0], inv_cols, a.eps));
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        const F2 r(rstd);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            F2 o[4], w[4], b[4];
            weight.get(i, w);
            bias.get(i, b);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = v[i][k] * r;
                o[k] = fma2(v[i][k], w[k], b[k]);
            }
            Eight<TYPE> out;
            out.set(o);
            store_eight<ALIGNED>(y + i * G * 8, out, n[i]);
            if (a.codes.codes) put_codes(a.codes, row, pitch, (i * G + t) * 8, v[i]);
        }
    }
}

// The backward pass in the same manner: dy and xhat are read once, a thread's columns
// of dw and db are added up in registers over the CTA's rows and go to
// work[CTA][2][cols], which novak_layer_norm_finish_kernel adds up in order.
template <int TYPE, int G, int NV, bool ALIGNED, bool FROM8>
__global__ void __launch_bounds__(32 * backward_warps<G, NV>(), G == 256 ? 2 : 1)
novak_layer_norm_back_kernel(NormBackArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[G == 32 ? 1 : 4 * 32];
    extern __shared__ __align__(16) float held[];       // warps: the weight, then the warps' column sums
    int turn = 0;
    const int t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0;
    constexpr int kWarps = backward_warps<G, NV>(), kSubs = G == 32 ? kWarps : 1;
    const int cols = static_cast<int>(a.cols), pitch = (cols + 31) / 32 * 32;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kSubs;
    const float inv_cols = 1.0f / static_cast<float>(cols);
    int64_t row = static_cast<int64_t>(blockIdx.x) * kSubs + sub;
    const T *dy = static_cast<const T *>(a.dy.ptr) + row * a.dy.stride + t * 8;
    const T *x = static_cast<const T *>(a.x.ptr) + row * a.x.stride + t * 8;
    const int8_t *codes = a.codes.codes + row * pitch + t * 8;
    const uint8_t *exps = a.codes.exps + row * (pitch / 32) + t / 4;
    T *dx = static_cast<T *>(a.dx.ptr) + row * a.dx.stride + t * 8;
    const void *dy_end = end_of(static_cast<const T *>(a.dy.ptr), a.dy.stride, a.rows, cols);
    const void *x_end = end_of(static_cast<const T *>(a.x.ptr), a.x.stride, a.rows, cols);
    int n[NV];
    Fetch<TYPE, ALIGNED> raw[NV], raw_x[FROM8 ? 1 : NV];
    uint2 q[FROM8 ? NV : 1];
    uint32_t e[FROM8 ? NV : 1];
    float rstd = 0.0f, mean = 0.0f;
    auto fetch = [&](int64_t at) {
        if (at >= a.rows) return;
        rstd = a.rstd[at];
        if (!FROM8) mean = a.mean[at];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].load(dy + i * G * 8, n[i], a.dy.ptr, dy_end);
            if constexpr (FROM8) {
                if (n[i] > 0) {
                    q[i] = *reinterpret_cast<const uint2 *>(codes + i * G * 8);
                    e[i] = exps[i * G / 4];
                }
            } else {
                raw_x[i].load(x + i * G * 8, n[i], a.x.ptr, x_end);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        n[i] = max(min(cols - (i * G + t) * 8, 8), 0);
        raw[i].zero();
        if constexpr (FROM8) {
            q[i] = make_uint2(0, 0);
            e[i] = 0;
        } else {
            raw_x[i].zero();
        }
    }
    start();
    fetch(row);
    Held<G, NV> weight;
    weight.load(a.weight, a.param_type, cols, held);
    if constexpr (G == 32) __syncthreads();
    F2 dw[NV][4], db[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[i][k] = db[i][k] = F2(0.0f);
    for (; row < a.rows; row += step, dx += step * a.dx.stride) {
        // (beyond the row dy, codes or x, and the weight are zeros: xhat is finite there)
        F2 g[NV][4], xh[NV][4], s0(0.0f), s1(0.0f);
        const float r = rstd;
        const F2 r2(r), m2(-mean);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i].eight().get(g[i]);
            if constexpr (FROM8) dequantize8(q[i], e[i], xh[i]);
            else raw_x[i].eight().get(xh[i]);
            F2 w[4];
            weight.get(i, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!FROM8) xh[i][k] = (xh[i][k] + m2) * r2;
                dw[i][k] = fma2(g[i][k], xh[i][k], dw[i][k]);
                db[i][k] = db[i][k] + g[i][k];
                g[i][k] = g[i][k] * w[k];
                s0 = s0 + g[i][k];
                s1 = fma2(g[i][k], xh[i][k], s1);
            }
        }
        dy += step * a.dy.stride;
        if constexpr (FROM8) {
            codes += step * pitch;
            exps += step * (pitch / 32);
        } else {
            x += step * a.x.stride;
        }
        fetch(row + step);
        float s[2] = {s0.lo() + s0.hi(), s1.lo() + s1.hi()};
        row_sums<G, 2>(s, scratch, turn);
        const F2 a1(-s[1] * inv_cols * r), a0(-s[0] * inv_cols * r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) g[i][k] = fma2(g[i][k], r2, fma2(xh[i][k], a1, a0));
            Eight<TYPE> out;
            out.set(g[i]);
            store_eight<ALIGNED>(dx + i * G * 8, out, n[i]);
        }
    }
    if (!a.dweight && !a.dbias) return;
    float *out = a.work + static_cast<int64_t>(blockIdx.x) * 2 * cols;
    if constexpr (G == 32) {
        float *part = held + NV * 256;
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const F2 lo = which ? db[i][2 * k] : dw[i][2 * k], hi = which ? db[i][2 * k + 1] : dw[i][2 * k + 1];
                    *reinterpret_cast<float4 *>(part + sub * NV * 256 + Held<G, NV>::at(i, 4 * k, t)) =
                        make_float4(lo.lo(), lo.hi(), hi.lo(), hi.hi());
                }
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += blockDim.x) {
                const int at = Held<G, NV>::at(c / 256, c % 8, c / 8 % 32);
                float sum = 0.0f;
#pragma unroll
                for (int p = 0; p < kWarps; ++p) sum += part[p * NV * 256 + at];
                out[which * cols + c] = sum;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int col = (i * G + t) * 8 + 2 * k;
                if (2 * k < n[i]) {
                    out[col] = dw[i][k].lo();
                    out[cols + col] = db[i][k].lo();
                }
                if (2 * k + 1 < n[i]) {
                    out[col + 1] = dw[i][k].hi();
                    out[cols + col + 1] = db[i][k].hi();
                }
            }
    }
}

// ---- rows too long for registers ---------------------------------------------------------
// One CTA per row, any length: the row is read three times (from L2 after the
// first time).
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_layer_norm_long_kernel(NormArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float scratch[33];
    start();
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
                F2 p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) p[k] = F2(v[2 * k], v[2 * k + 1]);
                put_codes(a.codes, row, pitch, c, p);
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
    start();
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
    start();
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

// dw, db from the partial sums: 32 columns of one of the two per CTA, each warp every
// 32nd sum in order, then the warps in order.
constexpr int kFinishThreads = 1024;
__global__ void __launch_bounds__(kFinishThreads)
novak_layer_norm_finish_kernel(const float *work, int64_t splits, int64_t cols, void *dweight, void *dbias, int type)
{
    __shared__ float part[32][33];
    start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, which = blockIdx.y;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    void *out = which ? dbias : dweight;
    if (!out) return;
    float sum = 0.0f;
    if (c < cols) {
        const float *src = work + which * cols + c;
#pragma unroll 8
        for (int64_t s = warp; s < splits; s += 32) sum += src[2 * s * cols];
    }
    part[lane][warp] = sum;
    __syncthreads();
    sum = warp_sum(part[warp][lane]);       // column `warp` of the 32
    const int64_t mine = static_cast<int64_t>(blockIdx.x) * 32 + warp;
    if (lane == 0 && mine < cols) store_param(out, type, mine, sum);
}

// How a row of `cols` elements is spread: G threads, NV groups of 8 each.  false: too
// long for registers.  Rows that are not aligned need more registers per group, and threads
// without elements cost what the others do (bf16, forward with the 8-bit form left and back:
// 12608 x 771 with 128 threads 25.5 and 27.1 us, with 512 112 and 84; 8000 x 2051 with 512 of one
// group 75 and 60, of two 100 and 105).
struct Spread {
    int g, nv;
};
constexpr Spread kAlignedRows[] = {{32, 1}, {32, 2}, {32, 3}, {32, 4}, {256, 1}, {256, 2}, {512, 2}};
constexpr Spread kAnyRows[] = {{32, 1}, {128, 1}, {512, 1}, {512, 2}};

template <int N> bool spread_for(const Spread (&from)[N], int64_t cols, Spread &s)
{
    for (const Spread &c : from)
        if (cols <= 8 * c.g * c.nv) {
            s = c;
            return true;
        }
    return false;
}

#define NOVAK_SPREADS(F)                                                                                          \
    F(32, 1, true) F(32, 2, true) F(32, 3, true) F(32, 4, true) F(256, 1, true) F(256, 2, true) F(512, 2, true) \
    F(32, 1, false) F(128, 1, false) F(512, 1, false) F(512, 2, false)

// CTAs of the backward pass, each of which leaves one partial sum per column: one per SM
// where its warps have a row each, else what hides a row's latency (12608 x 2048 bf16:
// one of 256 threads per SM 65 us, two 44, three 56, whose partial sums cost more than
// they hide; 8000 x 4096 bf16: one of 512 threads 54, two of 256 51; 12608 x 771 bf16, 128
// threads: two 36.7, four 27.1, eight 31.9).
int64_t back_ctas(const Spread &s, int64_t rows)
{
    const int per_sm = s.g == 32 || s.g == 512 ? 1 : s.g == 128 ? 4 : 2;
    return std::min<int64_t>(rows, kSms * per_sm);
}

// CTAs per SM of the forward pass: what registers leave room for (4096 columns: bf16
// 33 us with three of 256 threads, 39 with two of 512; fp32 29 and 30).  Rows that are not
// aligned: 12608 x 771 with four of 128 threads 27.6 us (fp32 42.6), with eight 25.5 (30.6), with
// twelve 25.5 (28.9); 8000 x 2051 with one of 512 73.9, two 74.9, three 75.9; 4000 x 7001, two
// groups per thread, with one 63.1, two 64.1.
constexpr int forward_ctas(int type, int g, int nv)
{
    return g == 32 ? 4 : g == 256 ? (nv == 1 ? 4 : type == NOVAK_TYPE_F32 ? 2 : 3) : 1024 / g / nv;
}

template <int TYPE> cudaError_t forward(const NormArgs &a, const Spread &s, bool aligned, cudaStream_t stream)
{
#define NOVAK_CASE(G, NV, ALIGNED)                                                                                    \
    if (s.g == G && s.nv == NV && aligned == ALIGNED) {                                                               \
        constexpr int warps = forward_warps<G, NV>(), rows = G == 32 ? warps : 1;                                     \
        const int64_t grid = std::min<int64_t>((a.rows + rows - 1) / rows, kSms * forward_ctas(TYPE, G, NV));         \
        return launch(novak_layer_norm_kernel<TYPE, G, NV, ALIGNED>, dim3(static_cast<unsigned>(grid)), 32 * warps,   \
                      0, stream, a);                                                                                  \
    }
    NOVAK_SPREADS(NOVAK_CASE)
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

template <int TYPE, bool FROM8>
cudaError_t backward(const NormBackArgs &a, const Spread &s, bool aligned, int64_t grid, cudaStream_t stream)
{
#define NOVAK_CASE(G, NV, ALIGNED)                                                                                    \
    if (s.g == G && s.nv == NV && aligned == ALIGNED) {                                                               \
        constexpr int warps = backward_warps<G, NV>(), smem = G == 32 ? (1 + warps) * NV * 256 * 4 : 0;               \
        static_assert(smem <= 40 * 1024, "48 KB without asking, less the kernel's own");                              \
        return launch(novak_layer_norm_back_kernel<TYPE, G, NV, ALIGNED, FROM8>, dim3(static_cast<unsigned>(grid)),   \
                      32 * warps, smem, stream, a);                                                                   \
    }
    NOVAK_SPREADS(NOVAK_CASE)
#undef NOVAK_CASE
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.x, a.type, a.rows) && wide(a.y, a.type, a.rows);
    const bool aligned = w && a.cols % 8 == 0;
    Spread s;
    if (aligned ? spread_for(kAlignedRows, a.cols, s) : spread_for(kAnyRows, a.cols, s))
        return a.type == NOVAK_TYPE_F32 ? forward<0>(a, s, aligned, stream) : forward<1>(a, s, aligned, stream);
    const int grid = static_cast<int>(std::min<int64_t>(a.rows, kSms * 8));
    auto kernel = a.type == NOVAK_TYPE_F32
                      ? (w ? novak_layer_norm_long_kernel<0, true> : novak_layer_norm_long_kernel<0, false>)
                      : (w ? novak_layer_norm_long_kernel<1, true> : novak_layer_norm_long_kernel<1, false>);
    return launch(kernel, dim3(static_cast<unsigned>(grid)), kThreads, 0, stream, a);
}

// Enough for either way of the backward pass: which one it is depends on alignment.
size_t layer_norm_backward_bytes(int64_t rows, int64_t cols)
{
    int64_t splits = (rows + kSplitRows - 1) / kSplitRows;
    Spread s;
    if (spread_for(kAnyRows, cols, s)) splits = std::max(splits, back_ctas(s, rows));
    if (spread_for(kAlignedRows, cols, s)) splits = std::max(splits, back_ctas(s, rows));
    return static_cast<size_t>(splits * 2 * cols) * sizeof(float);
}

cudaError_t launch_layer_norm_backward(const NormBackArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.dy, a.type, a.rows) && wide(a.dx, a.type, a.rows) &&
                   (!a.x.ptr || wide(a.x, a.type, a.rows));
    const bool sums = a.dweight || a.dbias, aligned = w && a.cols % 8 == 0;
    int64_t splits = 0;
    Spread s;
    if (a.rows == 0) {
    } else if (aligned ? spread_for(kAlignedRows, a.cols, s) : spread_for(kAnyRows, a.cols, s)) {
        splits = back_ctas(s, a.rows);
        const bool q = a.codes.codes != nullptr;
        const cudaError_t e = a.type == NOVAK_TYPE_F32 ? (q ? backward<0, true>(a, s, aligned, splits, stream) : backward<0, false>(a, s, aligned, splits, stream))
                                                       : (q ? backward<1, true>(a, s, aligned, splits, stream) : backward<1, false>(a, s, aligned, splits, stream));
        if (e != cudaSuccess) return e;
    } else {
        splits = (a.rows + kSplitRows - 1) / kSplitRows;
        const int t = a.type == NOVAK_TYPE_F32 ? 0 : 1;
        if (sums) {         // first: dx may be written over dy
            auto columns = t == 0 ? (w ? novak_layer_norm_columns_kernel<0, true> : novak_layer_norm_columns_kernel<0, false>)
                                  : (w ? novak_layer_norm_columns_kernel<1, true> : novak_layer_norm_columns_kernel<1, false>);
            const dim3 grid(static_cast<unsigned>((a.cols + kColsPerCta - 1) / kColsPerCta), static_cast<unsigned>(splits));
            const cudaError_t e = launch(columns, grid, kThreads, 0, stream, a);
            if (e != cudaSuccess) return e;
        }
        auto kernel = t == 0 ? (w ? novak_layer_norm_back_long_kernel<0, true> : novak_layer_norm_back_long_kernel<0, false>)
                             : (w ? novak_layer_norm_back_long_kernel<1, true> : novak_layer_norm_back_long_kernel<1, false>);
        const cudaError_t e = launch(kernel, dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kSms * 8))), kThreads, 0, stream, a);
        if (e != cudaSuccess) return e;
    }
    if (!sums) return cudaSuccess;
    return launch(novak_layer_norm_finish_kernel, dim3(static_cast<unsigned>((a.cols + 31) / 32), 2), kFinishThreads, 0, stream,
                  static_cast<const float *>(a.work), splits, a.cols, a.dweight, a.dbias, a.grad_type);
}

}  // namespace novak
