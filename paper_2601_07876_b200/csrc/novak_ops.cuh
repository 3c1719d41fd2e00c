// Device helpers of the training operators: eight consecutive elements of a row
// at a time, and the 8-bit form of activations.
#pragma once

#include <cuda_bf16.h>

#include "novak.h"
#include "novak_ops.h"

namespace novak {

// The operators' kernels are launched with programmatic stream serialization: a kernel's
// CTAs come to be, and set up what is theirs alone, while the kernel before drains (packing
// and unpacking 8192 x 4096 bf16 in a row: 32.3 us, 34.8 with plain launches; layer norm of
// 12608 x 768 and unpacking its form: 19.3 and 22.5).  Each of them starts with this: it
// waits for the kernel before, and only then lets the next one come.  The other way round
// the one after the next could start while what came before this one is still at work.
__device__ __forceinline__ void start()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = grid;
    lc.blockDim = dim3(static_cast<unsigned>(threads));
    lc.dynamicSmemBytes = static_cast<size_t>(smem);
    lc.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, kernel, static_cast<Params>(args)...);
}

template <int TYPE> struct Elem;
template <> struct Elem<NOVAK_TYPE_F32> { using T = float; };
template <> struct Elem<NOVAK_TYPE_BF16> { using T = __nv_bfloat16; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
// Element i of a vector of either type.
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

// Two fp32 numbers per instruction.
struct F2 {
    uint64_t v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit F2(float x) : F2(x, x) {}
    __device__ __forceinline__ void get(float &lo, float &hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
    __device__ __forceinline__ float lo() const { float a, b; get(a, b); return a; }
    __device__ __forceinline__ float hi() const { float a, b; get(a, b); return b; }
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b)
{
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(a.v) : "l"(b.v));
    return a;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b)
{
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(a.v) : "l"(b.v));
    return a;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}
// bf16 pair -> fp32 pair, and back (to nearest even)
__device__ __forceinline__ F2 widen(uint32_t w) { return F2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t narrow(F2 x)
{
    uint32_t r;
    float lo, hi;
    x.get(lo, hi);
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Elements [col, col + 8) of a row, zeros from `cols` on.  WIDE: the row is
// 16-byte aligned; col is a multiple of 8.  A group that the row's end cuts is
// read element by element either way.
template <bool WIDE>
__device__ __forceinline__ void load8(const float *row, int64_t col, int64_t cols, float (&v)[8])
{
    if (WIDE && col + 8 <= cols) {
        const float4 a = *reinterpret_cast<const float4 *>(row + col);
        const float4 b = *reinterpret_cast<const float4 *>(row + col + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? row[col + i] : 0.0f;
    }
}

template <bool WIDE>
__device__ __forceinline__ void load8(const __nv_bfloat16 *row, int64_t col, int64_t cols, float (&v)[8])
{
    if (WIDE && col + 8 <= cols) {
        const uint4 t = *reinterpret_cast<const uint4 *>(row + col);
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? to_float(row[col + i]) : 0.0f;
    }
}

template <bool WIDE>
__device__ __forceinline__ void store8(float *row, int64_t col, int64_t cols, const float (&v)[8])
{
    if (WIDE && col + 8 <= cols) {
        *reinterpret_cast<float4 *>(row + col) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(row + col + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = v[i];
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

template <bool WIDE>
__device__ __forceinline__ void store8(__nv_bfloat16 *row, int64_t col, int64_t cols, const float (&v)[8])
{
    if (WIDE && col + 8 <= cols) {
        *reinterpret_cast<uint4 *>(row + col) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]),
                                                           bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = __float2bfloat16_rn(v[i]);
    }
}

// Eight consecutive elements of a 16-byte aligned row, as they are in memory.
template <int TYPE> struct Eight;
template <> struct Eight<NOVAK_TYPE_BF16> {
    uint4 w;
    __device__ __forceinline__ void zero() { w = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(F2 (&v)[4]) const
    {
        v[0] = widen(w.x);
        v[1] = widen(w.y);
        v[2] = widen(w.z);
        v[3] = widen(w.w);
    }
    // `v` as it is stored; the bits of the largest magnitude of the eight
    __device__ __forceinline__ void set(const F2 (&v)[4]) { w = make_uint4(narrow(v[0]), narrow(v[1]), narrow(v[2]), narrow(v[3])); }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = w; }
    __device__ __forceinline__ uint32_t top() const
    {
        const uint32_t m = 0x7fff7fffu;
        const uint32_t t = __vmaxu2(__vmaxu2(w.x & m, w.y & m), __vmaxu2(w.z & m, w.w & m));
        return max(t << 16, t & 0xffff0000u);
    }
};
template <> struct Eight<NOVAK_TYPE_F32> {
    // as they were loaded: forming pairs here would wait for the load
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const float *p)
    {
        a = *reinterpret_cast<const float4 *>(p);
        b = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void get(F2 (&v)[4]) const
    {
        v[0] = F2(a.x, a.y);
        v[1] = F2(a.z, a.w);
        v[2] = F2(b.x, b.y);
        v[3] = F2(b.z, b.w);
    }
    __device__ __forceinline__ void set(const F2 (&v)[4])
    {
        a = make_float4(v[0].lo(), v[0].hi(), v[1].lo(), v[1].hi());
        b = make_float4(v[2].lo(), v[2].hi(), v[3].lo(), v[3].hi());
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<float4 *>(p) = a;
        *reinterpret_cast<float4 *>(p + 4) = b;
    }
    __device__ __forceinline__ uint32_t top() const
    {
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(x[i]) & 0x7fffffffu);
        return t;
    }
};

// Eight consecutive elements of any row, fetched as the aligned 16-byte pieces that hold
// them: `words` as they are in memory, the first element `skip` bytes in.  Only the
// first n elements count (0 to 8), the others read as zeros.  A piece that reaches
// beyond the matrix (of bytes begin to end) is fetched element by element.
template <int TYPE> struct AnyEight {
    using T = typename Elem<TYPE>::T;
    static constexpr int kSize = static_cast<int>(sizeof(T)), kPieces = kSize / 2 + 1;
    uint32_t words[4 * kPieces];
    int skip, n;
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 4 * kPieces; ++i) words[i] = 0;
        skip = n = 0;
    }
    __device__ __forceinline__ void load(const T *p, int count, const void *begin, const void *end)
    {
        n = count;
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        skip = static_cast<int>(at & 15u);
        const char *piece = reinterpret_cast<const char *>(at - skip);
        const int bytes = skip + n * kSize;
        if (n > 0 && (piece < begin || piece + (bytes + 15) / 16 * 16 > end)) {
            skip = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kSize == 4) {
                    words[i] = i < n ? __float_as_uint(p[i]) : 0u;
                } else {
                    const uint32_t x = i < n ? reinterpret_cast<const uint16_t *>(p)[i] : 0u;
                    words[i / 2] = i & 1 ? words[i / 2] | x << 16 : x;
                }
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (n > 0 && 16 * k < bytes) w = *reinterpret_cast<const uint4 *>(piece + 16 * k);
            words[4 * k] = w.x;
            words[4 * k + 1] = w.y;
            words[4 * k + 2] = w.z;
            words[4 * k + 3] = w.w;
        }
    }
    __device__ __forceinline__ Eight<TYPE> eight() const
    {
        constexpr int kWords = 2 * kSize;           // of eight elements
        uint32_t w[kWords + 4];
#pragma unroll
        for (int i = 0; i < kWords + 4; ++i) w[i] = words[i];
        if (skip & 8)
#pragma unroll
            for (int i = 0; i < kWords + 2; ++i) w[i] = w[i + 2];
        if (skip & 4)
#pragma unroll
            for (int i = 0; i < kWords + 1; ++i) w[i] = w[i + 1];
        Eight<TYPE> r;
        if constexpr (kSize == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (skip & 2) * 8);
            if (n < 8)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (2 * i >= n) w[i] = 0;
                    else if (2 * i + 1 >= n) w[i] &= 0xffffu;
                }
            r.w = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            if (n < 8)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= n) w[i] = 0;
            r.a = make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
            r.b = make_float4(__uint_as_float(w[4]), __uint_as_float(w[5]), __uint_as_float(w[6]), __uint_as_float(w[7]));
        }
        return r;
    }
};

// Stores the first n of eight elements of any row (p aligned to its element).  The
// warp's lanes have consecutive groups of one row and are all here; those with elements
// come first, and only the last of them may have fewer than eight.  What an aligned
// 16-byte piece holds of two neighbouring lanes goes out in one store; the pieces at
// the warp's ends, whose other elements are not here, go element by element.
__device__ __forceinline__ void store_any(__nv_bfloat16 *p, const Eight<NOVAK_TYPE_BF16> &v, int n)
{
    const int lane = threadIdx.x & 31, skip = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15u), head = (16 - skip) / 2;
    // words 0-3 of the lane before, 4-7 own; the piece starts skip bytes before word 4
    uint32_t w[8] = {0, 0, 0, 0, v.w.x, v.w.y, v.w.z, v.w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xffffffffu, w[4 + i], 1);
    // a piece that starts skip bytes before w[4]: word 4 - skip / 4 rounded up, then a half
    const int back = (skip + 3) / 4;                        // words
    uint32_t t[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const uint32_t a = i < 4 ? (back & 1 ? w[3 + i] : w[4 + i]) : (back & 1 ? w[7] : 0u);
        const uint32_t b = back & 1 ? w[1 + i] : w[2 + i];
        t[i] = back & 2 ? b : a;
    }
    if (back == 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) t[i] = w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __funnelshift_r(t[i], t[i + 1], (skip & 2) * 8);
    const bool full = n >= head && (skip == 0 || lane > 0);
    const int next_full = __shfl_down_sync(0xffffffffu, static_cast<int>(full), 1);
    if (full) *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(p) - skip) = make_uint4(t[0], t[1], t[2], t[3]);
    const int from = full ? head : 0, to = lane < 31 && next_full ? min(n, head) : n;
    if (from < to) {
        const uint32_t own[4] = {v.w.x, v.w.y, v.w.z, v.w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= from && i < to)
                reinterpret_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(i & 1 ? own[i / 2] >> 16 : own[i / 2]);
    }
}

__device__ __forceinline__ void store_any(float *p, const Eight<NOVAK_TYPE_F32> &v, int n)
{
    const int lane = threadIdx.x & 31, back = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15u) / 4, head = 4 - back;
    // elements 0-3: the last of the lane before; 4-11: own
    float w[12] = {0, 0, 0, 0, v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
    for (int i = 1; i < 4; ++i) w[i] = __shfl_up_sync(0xffffffffu, w[8 + i], 1);
    float t[8];         // two pieces, from `back` elements before the first
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = back & 1 ? w[3 + i] : w[4 + i], b = back & 1 ? w[1 + i] : w[2 + i];
        t[i] = back & 2 ? b : a;
    }
    const bool first = n >= head && (back == 0 || lane > 0), second = n >= head + 4;
    const int next_first = __shfl_down_sync(0xffffffffu, static_cast<int>(first), 1);
    if (first) *reinterpret_cast<float4 *>(p - back) = make_float4(t[0], t[1], t[2], t[3]);
    if (second) *reinterpret_cast<float4 *>(p - back + 4) = make_float4(t[4], t[5], t[6], t[7]);
    const bool next = lane < 31 && next_first && n == 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool done = i < head ? first : i < head + 4 ? second : next;
        if (i < n && !done) p[i] = w[4 + i];
    }
}

// The two behind one face.  ALIGNED: n is 0 or 8 (rows are 16-byte aligned and a
// multiple of 8 elements long).
template <int TYPE, bool ALIGNED> struct Fetch;
template <int TYPE> struct Fetch<TYPE, true> {
    using T = typename Elem<TYPE>::T;
    Eight<TYPE> x;
    __device__ __forceinline__ void zero() { x.zero(); }
    __device__ __forceinline__ void load(const T *p, int n, const void *, const void *)
    {
        if (n > 0) x.load(p);
    }
    __device__ __forceinline__ const Eight<TYPE> &eight() const { return x; }
};
template <int TYPE> struct Fetch<TYPE, false> {
    using T = typename Elem<TYPE>::T;
    AnyEight<TYPE> x;
    __device__ __forceinline__ void zero() { x.zero(); }
    __device__ __forceinline__ void load(const T *p, int n, const void *begin, const void *end) { x.load(p, n, begin, end); }
    __device__ __forceinline__ Eight<TYPE> eight() const { return x.eight(); }
};
template <bool ALIGNED, int TYPE>
__device__ __forceinline__ void store_eight(typename Elem<TYPE>::T *p, const Eight<TYPE> &v, int n)
{
    if constexpr (ALIGNED) {
        if (n > 0) v.store(p);
    } else {
        store_any(p, v, n);
    }
}

// Address behind a matrix's last element.
template <typename T> __device__ __forceinline__ const void *end_of(const T *p, int64_t stride, int64_t rows, int64_t cols)
{
    return p + (rows - 1) * stride + cols;
}

// Exponent byte of a block whose largest magnitude has these bits (an infinity or
// NaN: 255), and the reciprocal of its scale.
__device__ __forceinline__ uint32_t block_exp(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : max(e, 6u) - 6u;
}
__device__ __forceinline__ float inverse_scale(uint32_t exp)
{
    return __uint_as_float((254u - (exp == 255u ? 254u : exp)) << 23);
}
// 128 scales is the next exponent's; what rounds to it is held at 127.  Below this
// mantissa nothing does.
__device__ __forceinline__ bool may_clamp(uint32_t top) { return (top & 0x7fffffu) >= 0x7f0000u; }

// x * 2^k + 1.5 * 2^23 is rounded once, to nearest even, at the units' place, where
// the sum's low byte is the code in two's complement.
constexpr float kMagic = 12582912.0f;

// The 8-bit form of eight elements; the four threads of a quad (lanes 4i..4i+3,
// all of which have to be here) hold one block of 32.  `top`: the bits of the
// largest magnitude of the eight.  Magnitudes compare as integers, infinities above
// all numbers and NaNs above those.
__device__ __forceinline__ uint2 quantize8(const F2 (&v)[4], uint32_t top, uint32_t &exp)
{
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    exp = block_exp(top);
    const F2 inv(inverse_scale(exp)), magic(kMagic);
    float b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) fma2(v[i], inv, magic).get(b[2 * i], b[2 * i + 1]);
    if (may_clamp(top)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = fminf(fmaxf(b[i], kMagic - 127.0f), kMagic + 127.0f);
    }
    uint32_t q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        q[i] = __byte_perm(__byte_perm(__float_as_uint(b[4 * i]), __float_as_uint(b[4 * i + 1]), 0x0040),
                           __byte_perm(__float_as_uint(b[4 * i + 2]), __float_as_uint(b[4 * i + 3]), 0x0040), 0x5410);
    return exp == 255u ? make_uint2(0u, 0u) : make_uint2(q[0], q[1]);
}

// Bits of the largest magnitude of eight numbers, a NaN's if one is among them.
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ uint32_t top_of(const F2 (&v)[4])
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i].get(x[2 * i], x[2 * i + 1]);
    return __float_as_uint(larger(larger(larger(x[0], x[1]), larger(x[2], x[3])), larger(larger(x[4], x[5]), larger(x[6], x[7]))));
}

__device__ __forceinline__ float scale_of(uint32_t exp)
{
    return exp ? __uint_as_float(exp << 23) : __uint_as_float(0x00400000u);
}

// What eight codes with this exponent byte stand for.  An exponent of 0 means
// 2^-127; 255 gives an infinite scale, which makes NaNs of codes of 0.
__device__ __forceinline__ void dequantize8(uint2 codes, uint32_t exp, F2 (&v)[4])
{
    const F2 scale(scale_of(exp)), offset(-8388736.0f);
    const uint32_t w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // the floats 2^23 + (code + 128), built from their bits
        const uint32_t lo = __byte_perm(w[i / 2], 0x4b000000u, i & 1 ? 0x7442 : 0x7440);
        const uint32_t hi = __byte_perm(w[i / 2], 0x4b000000u, i & 1 ? 0x7443 : 0x7441);
        v[i] = (F2(__uint_as_float(lo), __uint_as_float(hi)) + offset) * scale;
    }
}
__device__ __forceinline__ void dequantize8(uint2 codes, uint32_t exp, float (&v)[8])
{
    F2 p[4];
    dequantize8(codes, exp, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i].get(v[2 * i], v[2 * i + 1]);
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}

// Sum over the CTA's threads, the same in each; `scratch` holds 33 floats and may
// be used again after the next barrier.
__device__ __forceinline__ float block_sum(float x, float *scratch)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = (blockDim.x + 31) >> 5;
    x = warp_sum(x);
    __syncthreads();
    if (lane == 0) scratch[warp] = x;
    __syncthreads();
    return warp_sum(lane < n ? scratch[lane] : 0.0f);
}

}  // namespace novak
