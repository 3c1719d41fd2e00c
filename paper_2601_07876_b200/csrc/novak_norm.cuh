// What the layer norm's and the root-mean-square norm's kernels share: how a row is spread
// over threads, sums over it, the weight's columns, and the last sums of the columns.
#pragma once

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

// dw (and db: a partial sum has `vectors` of them, one behind the other) from the partial
// sums: 32 columns of one of them per CTA, each warp every 32nd sum in order, then the warps
// in order.
constexpr int kFinishThreads = 1024;
__global__ void __launch_bounds__(kFinishThreads)
novak_layer_norm_finish_kernel(const float *work, int64_t splits, int64_t cols, int vectors, void *dweight,
                               void *dbias, int type)
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
        for (int64_t s = warp; s < splits; s += 32) sum += src[vectors * s * cols];
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
#define NOVAK_SPREADS(F)                                                                                          \
    F(32, 1, true) F(32, 2, true) F(32, 3, true) F(32, 4, true) F(256, 1, true) F(256, 2, true) F(512, 2, true) \
    F(32, 1, false) F(128, 1, false) F(512, 1, false) F(512, 2, false)

template <int N> bool spread_for(const Spread (&from)[N], int64_t cols, Spread &s)
{
    for (const Spread &c : from)
        if (cols <= 8 * c.g * c.nv) {
            s = c;
            return true;
        }
    return false;
}

}  // namespace
}  // namespace novak
