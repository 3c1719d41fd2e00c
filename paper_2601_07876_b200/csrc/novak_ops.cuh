// Device helpers of the training operators: eight consecutive elements of a row
// at a time, and the 8-bit form of activations.
#pragma once

#include <cuda_bf16.h>

#include "novak.h"
#include "novak_ops.h"

namespace novak {

template <int TYPE> struct Elem;
template <> struct Elem<NOVAK_TYPE_F32> { using T = float; };
template <> struct Elem<NOVAK_TYPE_BF16> { using T = __nv_bfloat16; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x)
{
    return __float2bfloat16_rn(x);
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

// The 8-bit form of eight elements; the four threads of a quad (lanes 4i..4i+3,
// all of which have to be here) hold one block of 32.  Returns the block's
// exponent byte and the eight codes.
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], uint32_t &exp)
{
    // Magnitudes compare as integers, infinities above all numbers and NaNs
    // above those: one maximum finds the exponent and what cannot be held.
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = top >> 23;
    if (e == 255u) {
        exp = 255u;
        return make_uint2(0u, 0u);
    }
    exp = max(e, 6u) - 6u;
    const float inv = __uint_as_float((254u - exp) << 23);
    // x * 2^k + 1.5 * 2^23 is rounded once, to nearest even, at the units' place,
    // where the sum's low byte is the code in two's complement.
    constexpr float kMagic = 12582912.0f;
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        b[i] = __float_as_uint(fminf(fmaxf(fmaf(v[i], inv, kMagic), kMagic - 127.0f), kMagic + 127.0f));
    const uint32_t lo = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    const uint32_t hi = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    return make_uint2(lo, hi);
}

// What eight codes with this exponent byte stand for.  An exponent of 0 means
// 2^-127; 255 gives an infinite scale, which makes NaNs of codes of 0.
__device__ __forceinline__ void dequantize8(uint2 codes, uint32_t exp, float (&v)[8])
{
    const float scale = exp ? __uint_as_float(exp << 23) : __uint_as_float(0x00400000u);
    const uint32_t w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // the float 2^23 + (code + 128), built from its bits
        const uint32_t bits = __byte_perm(w[i / 4], 0x4b000000u, 0x7440 | (i & 3));
        v[i] = (__uint_as_float(bits) - 8388736.0f) * scale;
    }
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
