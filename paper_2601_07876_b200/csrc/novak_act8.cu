// The 8-bit form of activations (packing, unpacking) and the activation functions
// that leave it and take it up:
//     E = max(exponent(max |x| of 32) - 6, 0), s = 2^(E - 127), q = clamp(rint(x / s));
//     a = f(u), du = da f'(s q).
// One element costs one read and one write of everything it has.  A thread has eight
// neighbouring elements, a quad of lanes a block of 32, so that loads and stores are of
// 16 bytes and a block's maximum is two shuffles; two such groups per thread, both loaded
// first.  Bound by HBM where rows are 16-byte aligned: 8192 x 4096 bf16 packed in 15.8 us
// (6.42 TB/s) and unpacked in 14.8 (6.86, some of it out of L2); 12608 x 3072 bf16 through
// GELU with both forms left in 39.5 us (5.95 TB/s), back in 30.2 (6.46).  Rows that are
// not aligned are bound by the shifting of what they load and store, 410 instructions
// per warp and group of 8 at 77 % of the issue slots: 12608 x 3071 bf16 72 and 65 us,
// 8192 x 4095 packed in 26.8, unpacked in 29.8.  A small matrix is a launch: 197 x 1000
// fp32 2.1 and 2.4 us.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;
constexpr int kIdentity = -1;
constexpr int kUnroll = 2;          // groups of 8 per thread, all loads first

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

// Phi(-|u|) and exp(-u^2/2), Phi the normal distribution function, for bf16: by formula
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

// The same and Phi(u) for fp32, which that formula leaves twice as far off as erf in fp32
// does.  Below |u| = 1, Phi = 1/2 + u q(u^2); above, Phi(-|u|) = t p(t) exp(-u^2/2) with t = 1 /
// (1 + 0.3 |u|), as there, one degree more.  q and p are least-maximum fits by reweighted
// least squares, with the coefficients rounded one after the other: Phi is off by at most 9e-9
// and 3e-9 (and 4e-6 of the tail) beside the arithmetic.  12608 x 3072 fp32 stays bound by
// HBM (59 us, back 52); on rows that are not aligned it takes 7 us of 84 more than the formula
// above, erff 15 and erfcf 37.
__device__ __forceinline__ F2 below_one(F2 u, F2 small, F2 large)
{
    return F2(fabsf(u.lo()) < 1.0f ? small.lo() : large.lo(), fabsf(u.hi()) < 1.0f ? small.hi() : large.hi());
}
__device__ __forceinline__ void normal_f32(F2 u, F2 &minus_mag, F2 &tail, F2 &cdf, F2 &e)
{
    const F2 mag(fabsf(u.lo()), fabsf(u.hi())), sq = u * u;
    minus_mag = mag * F2(-1.0f);
    const F2 t = rcp_approx(fma2(mag, F2(0.3f), F2(1.0f)));
    e = exp2_approx(sq * F2(-0.5f * 1.44269504f));
    F2 p = fma2(t, F2(-0.08579722f), F2(0.24261388f));
    p = fma2(p, t, F2(-0.04816293f));
    p = fma2(p, t, F2(0.16174269f));
    p = fma2(p, t, F2(0.109038524f));
    p = fma2(p, t, F2(0.120554216f));
    const F2 far = p * t * e, rest = fma2(far, F2(-1.0f), F2(1.0f));
    F2 q = fma2(sq, F2(9.2202055e-05f), F2(-0.001164883f));
    q = fma2(q, sq, F2(0.009963931f));
    q = fma2(q, sq, F2(-0.066488706f));
    q = fma2(q, sq, F2(0.3989422f));
    tail = below_one(u, fma2(minus_mag, q, F2(0.5f)), far);
    cdf = below_one(u, fma2(u, q, F2(0.5f)),
                    F2(u.lo() > 0.0f ? rest.lo() : far.lo(), u.hi() > 0.0f ? rest.hi() : far.hi()));
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

template <int KIND, int TYPE>
__device__ __forceinline__ F2 act(F2 u)
{
    if constexpr (KIND == NOVAK_ACT_GELU) {
        F2 minus_mag, tail, cdf, e;
        if constexpr (TYPE == NOVAK_TYPE_F32) {
            normal_f32(u, minus_mag, tail, cdf, e);
        } else {
            normal_tail(u, minus_mag, tail, e);
            minus_mag = minus_mag * F2(-1.0f);
        }
        // u (1 - tail) above zero, u tail below
        return fma2(minus_mag, tail, F2(fmaxf(u.lo(), 0.0f), fmaxf(u.hi(), 0.0f)));
    }
    if constexpr (KIND == NOVAK_ACT_GELU_TANH) return u * logistic(tanh_argument(u));
    if constexpr (KIND == NOVAK_ACT_SILU) return u * logistic(u * F2(-kLog2e));
    return u;
}

// GELU's tail times an infinity is a NaN, which for plus infinity is not f's value.  Looked
// for where the largest magnitude of the eight says so; a bound on each |u| costs 4 % of a
// kernel that instructions bound (rows that are not aligned).
constexpr uint32_t kInfinityBits = 0x7f800000u;
__device__ __forceinline__ void put_infinities(const F2 (&u)[4], F2 (&f)[4])
{
    const float inf = __uint_as_float(kInfinityBits);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        f[k] = F2(u[k].lo() == inf ? inf : f[k].lo(), u[k].hi() == inf ? inf : f[k].hi());
}

template <int KIND, int TYPE>
__device__ __forceinline__ F2 act_slope(F2 u)
{
    if constexpr (KIND == NOVAK_ACT_GELU) {
        F2 mag, tail, e, cdf;
        if constexpr (TYPE == NOVAK_TYPE_F32) {
            normal_f32(u, mag, tail, cdf, e);
        } else {
            normal_tail(u, mag, tail, e);
            const F2 h = fma2(tail, F2(-1.0f), F2(0.5f));   // Phi(u) = 1/2 +- h
            cdf = F2(copysignf(h.lo(), u.lo()), copysignf(h.hi(), u.hi())) + F2(0.5f);
        }
        return fma2(u * F2(0.39894228f), e, cdf);
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

// Where a thread's eight elements are.  FLAT: rows without gaps, a multiple of 32 long,
// are one run of elements.  Otherwise 2^log2 neighbouring threads (a warp at least)
// share a row.
struct Place {
    int64_t rows, cols;
    int64_t groups;         // of 8 elements: all of them (FLAT), or of a row's pitch
    int log2;
};

struct At {
    int64_t row, col;       // FLAT: row 0, col over the whole run
    bool in;                // inside the rows and their padding
    int n;                  // elements of the row, 0 to 8
};

template <bool FLAT>
__device__ __forceinline__ At place(const Place &p, int64_t first_row, int u)
{
    if constexpr (FLAT) {
        const int64_t g = (static_cast<int64_t>(blockIdx.x) * kUnroll + u) * kThreads + threadIdx.x;
        const bool in = g < p.groups;
        return {0, g * 8, in, in ? 8 : 0};
    } else {
        const int64_t g = (static_cast<int64_t>(blockIdx.x) << p.log2) + (threadIdx.x & ((1 << p.log2) - 1));
        const int64_t row = first_row + (static_cast<int64_t>(u) << (8 - p.log2)) + (threadIdx.x >> p.log2);
        const bool in = g < p.groups && row < p.rows;
        return {row, g * 8, in, in ? static_cast<int>(max(min(p.cols - g * 8, int64_t(8)), int64_t(0))) : 0};
    }
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

// Flat rows are aligned; others may be.
enum Rows { kFlat, kAligned, kAny };

// bf16 in one run is held to 32 registers, with which every thread that an SM has room for
// is there: GELU of 12608 x 3072 39.5 us, 40.2 with those that it would take.  (0: no bound.)
template <int KIND, int TYPE, Rows ROWS>
__global__ void __launch_bounds__(kThreads, TYPE == NOVAK_TYPE_BF16 && ROWS == kFlat ? 2048 / kThreads : 0)
novak_activation_kernel(const typename Elem<TYPE>::T *u, int64_t u_stride, typename Elem<TYPE>::T *a, int64_t a_stride,
                        Codes uc, Codes ac, Place p)
{
    constexpr bool kIsFlat = ROWS == kFlat, kIsAligned = ROWS != kAny;
    const int64_t pitch = (p.cols + 31) / 32 * 32;
    const int64_t per_pass = kIsFlat ? 1 : int64_t(kUnroll) << (8 - p.log2);
    const void *end = end_of(u, u_stride, p.rows, p.cols);
    start();
    for (int64_t row0 = blockIdx.y * per_pass; row0 < (kIsFlat ? 1 : p.rows); row0 += gridDim.y * per_pass) {
        Fetch<TYPE, kIsAligned> raw[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<kIsFlat>(p, row0, i);
            raw[i].zero();
            raw[i].load(u + at.row * u_stride + at.col, at.n, u, end);
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<kIsFlat>(p, row0, i);
            const int64_t to = at.row * pitch + at.col;
            const Eight<TYPE> x = raw[i].eight();
            F2 v[4];
            x.get(v);
            const uint32_t top = x.top();
            if (uc.codes) put(uc, to, at.in, v, top);
            if constexpr (KIND != kIdentity) {
                F2 f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = act<KIND, TYPE>(v[k]);
                if (KIND == NOVAK_ACT_GELU && top >= kInfinityBits) put_infinities(v, f);
                Eight<TYPE> out;
                out.set(f);
                if (a) store_eight<kIsAligned>(a + at.row * a_stride + at.col, out, at.n);
                if (ac.codes) {         // of what the next layer reads: the rounded values
                    out.get(f);         // (beyond the row f(0) = 0)
                    put(ac, to, at.in, f, out.top());
                }
            }
        }
    }
}

// fp32 from the 8-bit form on rows that are not aligned is held to 64 registers, four CTAs per
// SM: 12608 x 3071 GELU 91 us, 97 with the 66 that it would take; SiLU 76.6 and 80.7.  From u,
// SiLU is slower for it (98.7 and 92.8).
template <int KIND, int TYPE, Rows ROWS, bool FROM8>
__global__ void __launch_bounds__(kThreads, FROM8 && TYPE == NOVAK_TYPE_F32 && ROWS == kAny ? 4 : 0)
novak_activation_backward_kernel(const typename Elem<TYPE>::T *da, int64_t da_stride, const typename Elem<TYPE>::T *u,
                                 int64_t u_stride, Codes uc, typename Elem<TYPE>::T *du, int64_t du_stride, Place p)
{
    constexpr bool kIsFlat = ROWS == kFlat, kIsAligned = ROWS != kAny;
    const int64_t pitch = (p.cols + 31) / 32 * 32;
    const int64_t per_pass = kIsFlat ? 1 : int64_t(kUnroll) << (8 - p.log2);
    const void *da_end = end_of(da, da_stride, p.rows, p.cols), *u_end = end_of(u, u_stride, p.rows, p.cols);
    start();
    for (int64_t row0 = blockIdx.y * per_pass; row0 < (kIsFlat ? 1 : p.rows); row0 += gridDim.y * per_pass) {
        Fetch<TYPE, kIsAligned> raw[kUnroll], raw_u[FROM8 ? 1 : kUnroll];
        uint2 q[FROM8 ? kUnroll : 1];
        uint32_t e[FROM8 ? kUnroll : 1];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<kIsFlat>(p, row0, i);
            if (kIsAligned && at.n == 0) continue;
            if constexpr (KIND != kIdentity) {
                if (!kIsAligned) raw[i].zero();
                raw[i].load(da + at.row * da_stride + at.col, at.n, da, da_end);
            }
            if constexpr (FROM8) {
                const int64_t from = at.row * pitch + at.col;
                if (!kIsAligned) {
                    q[i] = make_uint2(0, 0);
                    e[i] = 0;
                }
                if (at.n > 0) {
                    q[i] = *reinterpret_cast<const uint2 *>(uc.codes + from);
                    e[i] = uc.exps[from >> 5];
                }
            } else {
                if (!kIsAligned) raw_u[i].zero();
                raw_u[i].load(u + at.row * u_stride + at.col, at.n, u, u_end);
            }
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const At at = place<kIsFlat>(p, row0, i);
            if (kIsAligned && at.n == 0) continue;
            F2 v[4];
            if constexpr (FROM8) dequantize8(q[i], e[i], v);
            else raw_u[i].eight().get(v);
            if constexpr (KIND != kIdentity) {
                F2 g[4];
                raw[i].eight().get(g);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = g[k] * act_slope<KIND, TYPE>(v[k]);
            }
            Eight<TYPE> out;
            out.set(v);
            store_eight<kIsAligned>(du + at.row * du_stride + at.col, out, at.n);
        }
    }
}

// The form that the matrices allow, and its grid.
Rows rows_of(const Mat &x, const Mat &y, const Mat &z, int type, Place &p, dim3 &grid)
{
    const Mat *all[3] = {&x, &y, &z};
    bool aligned = p.cols % 8 == 0, flat = p.cols % 32 == 0 && p.rows * p.cols < (int64_t(1) << 42);
    for (const Mat *m : all) {
        if (!m->ptr) continue;
        aligned = aligned && wide(*m, type, p.rows);
        flat = flat && (p.rows <= 1 || m->stride == p.cols);
    }
    if (aligned && flat) {
        p.groups = p.rows * p.cols / 8;
        grid = dim3(static_cast<unsigned>((p.groups + kThreads * kUnroll - 1) / (kThreads * kUnroll)));
        return kFlat;
    }
    p.groups = act_pitch(p.cols) / 8;
    p.log2 = 5;             // a warp is in one row; the most threads that leave the fewest over
    for (int i = 6; i <= 8; ++i)
        if ((-p.groups & ((int64_t(1) << i) - 1)) <= (-p.groups & 31)) p.log2 = i;
    const int64_t per_pass = int64_t(kUnroll) << (8 - p.log2);
    grid = dim3(static_cast<unsigned>((p.groups + (int64_t(1) << p.log2) - 1) >> p.log2),
                static_cast<unsigned>(std::min<int64_t>((p.rows + per_pass - 1) / per_pass, 65535)));
    return aligned ? kAligned : kAny;
}

template <int KIND, int TYPE>
cudaError_t forward(Mat u, Mat a, Codes uc, Codes ac, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    Place p{rows, cols, 0, 0};
    dim3 grid;
    const Rows r = rows_of(u, a, Mat{}, TYPE, p, grid);
    auto kernel = r == kFlat      ? novak_activation_kernel<KIND, TYPE, kFlat>
                  : r == kAligned ? novak_activation_kernel<KIND, TYPE, kAligned>
                                  : novak_activation_kernel<KIND, TYPE, kAny>;
    return launch(kernel, grid, kThreads, 0, stream, static_cast<const T *>(u.ptr), u.stride, static_cast<T *>(a.ptr), a.stride, uc, ac, p);
}

template <int KIND, int TYPE, bool FROM8>
cudaError_t backward(Mat da, Mat u, Codes uc, Mat du, int64_t rows, int64_t cols, cudaStream_t stream)
{
    using T = typename Elem<TYPE>::T;
    Place p{rows, cols, 0, 0};
    dim3 grid;
    const Rows r = rows_of(da, u, du, TYPE, p, grid);
    auto kernel = r == kFlat      ? novak_activation_backward_kernel<KIND, TYPE, kFlat, FROM8>
                  : r == kAligned ? novak_activation_backward_kernel<KIND, TYPE, kAligned, FROM8>
                                  : novak_activation_backward_kernel<KIND, TYPE, kAny, FROM8>;
    return launch(kernel, grid, kThreads, 0, stream, static_cast<const T *>(da.ptr), da.stride, static_cast<const T *>(u.ptr),
                  u.stride, uc, static_cast<T *>(du.ptr), du.stride, p);
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
