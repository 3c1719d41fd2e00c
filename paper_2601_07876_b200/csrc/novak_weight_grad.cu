// Weight and bias gradient of a linear layer from the 8-bit form of its input:
//     dW[n, k] = sum_t dy[t, n] x[t, k],   db[n] = sum_t dy[t, n].
//
// What a code stands for has 7 significant bits and is exact in bf16, so a bf16
// dy needs one bf16 product per term and loses nothing; an fp32 dy is cut into
// three bf16 parts ("planes") that add up to its 24 bits.  With a layer norm's
// weight and bias, h = xhat w + b, and
//     dW[n, k] = w_k sum_t dy[t, n] xhat[t, k] + b_k sum_t dy[t, n]:
// the products are those of xhat, and w and b come in behind the sum.
//
// novak_weight_grad_kernel: pairs of CTAs (two SMs' tensor cores on one 256 x 256
// tile, cta_group::2), each CTA with
//   warps 0-7    the tile out of tensor memory, added up in registers,
//   warps 8-15   codes -> bf16, from and to swizzled shared memory,
//   warps 16-19  codes by tensor copies, and exponent bytes,
//   warp 20      dy by tensor copies,
//   warp 21      the products (of the pair: in the leading CTA),
//   warps 22-23  sums of dy's columns.
//
// dy and x both have the summed dimension (rows) outermost, so both operands are
// "M-major" and neither is transposed.
//
// Work: whole tiles as long as every pair gets one; the rows of the tiles that
// are left over are cut evenly over all pairs, partial tiles going to a
// workspace that novak_weight_grad_finish_kernel adds up in a fixed order.
#include <algorithm>
#include <atomic>

#include "novak_ops.cuh"
#include "novak_tcgen05.cuh"

namespace novak {
namespace {

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

// ---- few rows: the outer products, in fp32 on the ordinary cores ----------------
constexpr int kFewRows = 16;
constexpr int kTile = 64, kDepth = 16, kPlainThreads = 256;

// A 64 x 64 tile per CTA, 4 x 4 products per thread.
template <int TYPE>
__global__ void __launch_bounds__(kPlainThreads) novak_weight_grad_few_kernel(WeightGradArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ float sdy[kDepth][kTile], sx[kDepth][kTile];
    const int64_t pitch = (a.n_in + 31) / 32 * 32;
    const int64_t n0 = static_cast<int64_t>(blockIdx.y) * kTile, k0 = static_cast<int64_t>(blockIdx.x) * kTile;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float acc[4][4] = {}, sum[4] = {};
    for (int i = threadIdx.x; i < kDepth * kTile; i += kPlainThreads) {
        const int64_t t = i / kTile, n = n0 + i % kTile;
        sdy[i / kTile][i % kTile] = t < a.rows && n < a.n_out
                                        ? to_float(static_cast<const T *>(a.dy.ptr)[t * a.dy.stride + n]) : 0.0f;
    }
    if (threadIdx.x < kDepth * kTile / 8) {
        const int64_t t = threadIdx.x / 8, k = k0 + threadIdx.x % 8 * 8;
        float v[8] = {};
        if (t < a.rows && k < pitch)
            dequantize8(*reinterpret_cast<const uint2 *>(a.codes.codes + t * pitch + k),
                        a.codes.exps[(t * pitch + k) >> 5], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sx[threadIdx.x / 8][threadIdx.x % 8 * 8 + i] = v[i];
    }
    __syncthreads();
    for (int d = 0; d < static_cast<int>(a.rows); ++d) {
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + ty * 4 + i;
        if (n >= a.n_out) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t k = k0 + tx + 16 * j;
            if (k >= a.n_in) continue;
            float v = acc[i][j];
            if (a.weight)
                v = fmaf(v, param_at(a.weight, a.param_type, k), param_at(a.bias, a.param_type, k) * sum[i]);
            store_param(a.dw, a.grad_type, n * a.n_in + k, v);
        }
        if (a.db && blockIdx.x == 0 && tx == 0) store_param(a.db, a.grad_type, n, sum[i]);
    }
}

// ---- dy as the tensor copies need it ---------------------------------------------
// [planes][rows][ld] bf16, ld a multiple of 8: a copy of a bf16 matrix whose rows
// are not 16-byte aligned, or the three parts of an fp32 one.  Each part is what
// is left cut to 8 bits toward zero (so that none rounds up to an infinity); an
// infinity or NaN is in the first part alone.
template <int TYPE>
__global__ void __launch_bounds__(256)
novak_weight_grad_planes_kernel(const typename Elem<TYPE>::T *dy, int64_t stride, __nv_bfloat16 *out, int64_t ld,
                                int64_t rows, int64_t cols)
{
    const int64_t groups = ld / 8, n = rows * groups, plane = rows * ld;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        float v[8];
        load8<false>(dy + row * stride, col, cols, v);
        __nv_bfloat16 *dst = out + row * ld + col;
        if constexpr (TYPE == NOVAK_TYPE_BF16) {
            store8<true>(dst, 0, 8, v);
        } else {
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                float part[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool finite = (__float_as_uint(v[k]) & 0x7f800000u) != 0x7f800000u;
                    part[k] = finite ? __uint_as_float(__float_as_uint(v[k]) & 0xffff0000u) : v[k];
                    v[k] = finite ? v[k] - part[k] : 0.0f;
                }
                store8<true>(dst + p * plane, 0, 8, part);
            }
        }
    }
}

// ---- the work, cut up --------------------------------------------------------------
constexpr int kTileN = 256, kTileK = 256;       // dW rows and columns of a pair
constexpr int kRows = 64;                       // rows of dy and x per step
constexpr int kGroupN = 8;                      // tiles whose x is shared by neighbours in time
constexpr int kMinSteps = 4;                    // steps that are worth a pair's while

struct Cut {
    int tiles_n, tiles_k;
    int planes;
    int steps;              // of a tile: planes x ceil(rows / 64)
    int pairs;              // that run whole tiles
    int waves;              // whole tiles per pair
    int rest;               // tiles left over, after the first waves * pairs
    int rest_pairs;         // pairs among which their steps are cut
    int all_partial;        // every tile goes through the workspace
};

struct Piece {
    int tile;
    int first, count;       // steps
    int slot;               // of partial sums in the workspace
    bool whole;
};

// Steps [i] of the tiles left over that pair p starts with.
__host__ __device__ __forceinline__ int64_t rest_start(const Cut &c, int p)
{
    return static_cast<int64_t>(c.steps) * c.rest * p / c.rest_pairs;
}

__host__ __device__ __forceinline__ int slots(const Cut &c) { return c.rest_pairs + c.rest + c.tiles_n * c.tiles_k; }

struct Walk {
    const Cut &c;
    int pair, wave = 0;
    int64_t pos = 0, end = 0;
    __device__ Walk(const Cut &cut, int p) : c(cut), pair(p)
    {
        if (c.rest > 0 && p < c.rest_pairs) {
            pos = rest_start(c, p);
            end = rest_start(c, p + 1);
        }
    }
    __device__ bool next(Piece &p)
    {
        if (wave < c.waves) {
            p.tile = wave * c.pairs + pair;
            p.first = 0;
            p.count = c.steps;
            ++wave;
        } else if (pos < end) {
            const int r = static_cast<int>(pos / c.steps);
            p.tile = c.waves * c.pairs + r;
            p.first = static_cast<int>(pos - static_cast<int64_t>(r) * c.steps);
            p.count = static_cast<int>(min(static_cast<int64_t>(c.steps - p.first), end - pos));
            p.slot = pair + r;          // one more than the piece before has, or two
            pos += p.count;
        } else {
            return false;
        }
        p.whole = p.count == c.steps;
        if (p.whole) p.slot = c.rest_pairs + c.rest + p.tile;
        return true;
    }
};

// A step's 64 rows and its plane of dy; the planes of the same rows follow one another.
struct StepPos {
    int chunk, plane;
    __device__ __forceinline__ StepPos(const Cut &c, int step) : chunk(step / c.planes), plane(step - chunk * c.planes) {}
    __device__ __forceinline__ void advance(const Cut &c)
    {
        if (++plane == c.planes) {
            plane = 0;
            ++chunk;
        }
    }
};

// Tiles in groups of kGroupN tile rows, down the rows first.
__device__ __forceinline__ void tile_at(const Cut &c, int tile, int &tn, int &tk)
{
    const int per_group = kGroupN * c.tiles_k, g = tile / per_group, rows = min(kGroupN, c.tiles_n - g * kGroupN);
    const int in = tile - g * per_group;
    tk = in / rows;
    tn = g * kGroupN + in - tk * rows;
}

__device__ __forceinline__ int tile_index(const Cut &c, int tn, int tk)
{
    const int g = tn / kGroupN, rows = min(kGroupN, c.tiles_n - g * kGroupN);
    return g * kGroupN * c.tiles_k + tk * rows + tn - g * kGroupN;
}

// First slot and number of slots of a tile's partial sums (consecutive).
__device__ __forceinline__ void tile_slots(const Cut &c, int tile, int &slot, int &n)
{
    const int r = tile - c.waves * c.pairs;
    slot = c.rest_pairs + c.rest + tile;
    n = 1;
    if (r < 0) return;
    const int64_t steps = c.steps, total = steps * c.rest;
    // the pair that has step i: the last p with total p / rest_pairs <= i
    const int lo = static_cast<int>((static_cast<int64_t>(c.rest_pairs) * (r * steps + 1) - 1) / total);
    const int hi = static_cast<int>((static_cast<int64_t>(c.rest_pairs) * ((r + 1) * steps) - 1) / total);
    if (lo == hi) return;
    slot = lo + r;
    n = hi - lo + 1;
}

// ---- the kernel ----------------------------------------------------------------------
constexpr int kDySlots = 6, kXSlots = 3, kRawSlots = 8;         // steps of dy, of x, of codes
constexpr int kHalf = 64 * kRows * 2;                   // 64 columns of an operand, bf16
constexpr int kSlotBytes = 2 * kHalf;                   // 128 columns
constexpr int kRawBytes = 128 * kRows;                  // codes of 128 columns
constexpr int kRun = 16;        // steps that the tensor cores add up by themselves: their sums round toward
                                // zero, so that a chain's error grows with its length
constexpr int kOutWarps = 8, kFillWarps = 8, kFillGroups = 2, kLoadWarps = 4, kSumWarps = 2;
constexpr int kGroupWarps = kFillWarps / kFillGroups;   // that fill a step's x; the groups take turns
constexpr int kLoadWarp = kOutWarps + kFillWarps, kCopyWarp = kLoadWarp + kLoadWarps, kMmaWarp = kCopyWarp + 1,
              kSumWarp = kCopyWarp + 2;
constexpr int kThreads = 32 * (kSumWarp + kSumWarps);
// A barrier's parity tells one phase from the next, not from the one after that: whoever
// waits for a slot's use number k has to know that use k - 1 is over.  The two groups do
// not finish steps in order among each other, so a slot of codes belongs to one group for
// good; the products free the slots of dy and x in order.
static_assert(kRawSlots % kFillGroups == 0 && kRawSlots % kLoadWarps == 0, "slots of codes change hands");
static_assert(kXSlots <= kDySlots, "a step's end is kept for as long as dy's slots last");
constexpr int kPad = 9;
// Registers per thread: 80 at launch, 768 x 80 = 61440 = 256 x 160 + 512 x 40.
constexpr int kOutRegs = 160, kOtherRegs = 40;

struct Shared {
    alignas(8) uint64_t dy_full[kDySlots], full[kXSlots], filled[kXSlots], raw_full[kRawSlots], raw_empty[kRawSlots], out_full[2], out_empty[2],
        drained;
    uint64_t done[kDySlots];            // a step's products are over: step i's is done[i % kDySlots]
    uint32_t tmem;
    uint32_t exps[kRawSlots][kRows];    // of four blocks
    float turn[kOutWarps][32 * kPad];
};
constexpr int kSmemBytes = (kDySlots + kXSlots) * kSlotBytes + kRawSlots * kRawBytes + 1024 + static_cast<int>(sizeof(Shared));
static_assert(kSmemBytes <= 227 * 1024, "shared memory");

// A position in a ring of N slots, and the parity of its use.
template <int N> struct Ring {
    uint32_t slot, phase = 0;
    __device__ explicit Ring(uint32_t first = 0) : slot(first) {}
    __device__ __forceinline__ void advance(int n = 1)
    {
        slot += n;
        if (slot >= N) {
            slot -= N;
            phase ^= 1;
        }
    }
};

struct KernelArgs {
    Cut cut;
    Codes codes;
    int64_t pitch;
    void *dw;
    int grad_type, vector;
    int64_t rows, n_out, n_in;
    float *partial;                 // [slot][64][256 rows][4 columns] per tile
    float *sums;                    // [slot][256]; NULL: not asked for
};

__device__ unsigned g_gave_up;       // warps whose wait for a tile ran out, since the library was loaded

// Sixteen codes -> bf16, exactly: |code| and sign as bf16 numbers 128 + low bits and
// 128 or 256, whose difference is the code; then the scale, a power of two.
__device__ __forceinline__ void codes_to_bf16(const uint32_t (&w)[4], uint32_t s2, uint32_t (&out)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t p = __byte_perm(w[i / 2], 0x43434343u, i & 1 ? 0x4342 : 0x4140);
        const uint32_t low = p & 0xff7fff7fu, high = p & 0xff80ff80u;
        const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&low),
                                                 *reinterpret_cast<const __nv_bfloat162 *>(&high)),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&s2));
        out[i] = *reinterpret_cast<const uint32_t *>(&v);
    }
}

// Warps kLoadWarp ..: the 64 x 128 codes of a step by a tensor copy, and their
// exponent bytes; each warp has every fourth step.
__device__ __forceinline__ void load_codes(const KernelArgs &a, const CUtensorMap *map, Shared &sh, uint32_t raws,
                                           uint32_t rank, int pair)
{
    const int mine = threadIdx.x / 32 - kLoadWarp, lane = threadIdx.x % 32;
    const int64_t blocks = a.pitch / 32;
    const bool words = (blocks & 3) == 0 && (reinterpret_cast<uintptr_t>(a.codes.exps) & 3) == 0;
    Walk walk(a.cut, pair);
    Piece piece;
    Ring<kRawSlots> raw, last;
    uint32_t step = 0;
    bool any = false;
    while (walk.next(piece)) {
        int tn, tk;
        tile_at(a.cut, piece.tile, tn, tk);
        StepPos at(a.cut, piece.first);
        const int64_t block0 = static_cast<int64_t>(tk) * (kTileK / 32) + rank * 4;
        for (int i = 0; i < piece.count; ++i, ++step, at.advance(a.cut)) {
            if (step % kLoadWarps == mine) {
                if (!mbar_wait_warp(smem_addr(&sh.raw_empty[raw.slot]), raw.phase ^ 1)) {
                    if (any) mbar_wait_warp(smem_addr(&sh.raw_full[last.slot]), last.phase);      // its copy in flight
                    return;
                }
                last = raw;
                any = true;
                const uint32_t bar = smem_addr(&sh.raw_full[raw.slot]);
                if (lane == 0) {
                    mbar_expect(bar, kRawBytes);
                    tma_load_2d(raws + raw.slot * kRawBytes, map, static_cast<int>(block0) * 32, at.chunk * kRows, bar);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t row = static_cast<int64_t>(at.chunk) * kRows + lane + 32 * h;
                    uint32_t e = 0;
                    if (row < a.rows) {
                        const uint8_t *src = a.codes.exps + row * blocks + block0;
                        if (words) {
                            if (block0 < blocks) e = __ldg(reinterpret_cast<const uint32_t *>(src));
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (block0 + k < blocks) e |= static_cast<uint32_t>(__ldg(src + k)) << (8 * k);
                        }
                    }
                    sh.exps[raw.slot][lane + 32 * h] = e;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);
            }
            raw.advance();
        }
    }
}

// Warps kOutWarps ..: x, 64 rows x 128 columns per step, a thread one block of each of
// two rows.  The eight threads of a shared-memory access have eight consecutive rows,
// which the 128-byte swizzle spreads over all banks, of the codes and of x.  Two groups
// of four warps have every other step each: a step's waits, its proxy fence and its
// arrival take longer than its arithmetic.
__device__ __forceinline__ void fill_x(const KernelArgs &a, Shared &sh, uint32_t xs, uint32_t raws, uint32_t rank, int pair)
{
    const int group = (threadIdx.x / 32 - kOutWarps) / kGroupWarps, warp = (threadIdx.x / 32 - kOutWarps) % kGroupWarps;
    const int lane = threadIdx.x % 32, half = warp & 1, r = (warp >> 1) * 32 + (lane & 15), b = lane >> 4;
    const uint32_t dst0 = xs + half * kHalf + r * 128 + ((4 * b ^ (r & 7)) << 4);
    const uint32_t src0 = raws + r * 128 + (((half * 4 + b * 2) ^ (r & 7)) << 4);
    const uint32_t exp0 = smem_addr(&sh.exps[0][0]) + r * 4 + half * 2 + b;
    int steps = 0;
    {
        Walk count(a.cut, pair);
        Piece piece;
        while (count.next(piece)) steps += piece.count;
    }
    Ring<kXSlots> x(group);
    Ring<kRawSlots> raw(group);
    Ring<kDySlots> before(kDySlots + group - kXSlots);      // the step that had x's slot before
    before.phase = 1;
    const uint32_t done = smem_addr(&sh.done[0]), filled = smem_addr(rank == 0 ? &sh.full[0] : &sh.filled[0]);
    const uint32_t raw_full = smem_addr(&sh.raw_full[0]), raw_empty = smem_addr(&sh.raw_empty[0]);
    for (int step = group; step < steps; step += kFillGroups) {
        if (!mbar_wait_warp(raw_full + raw.slot * 8, raw.phase)) return;
        uint32_t q[4][4], e[2];
        const uint32_t src = src0 + raw.slot * kRawBytes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e[k]) : "r"(exp0 + raw.slot * (kRows * 4) + k * 64));
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[2 * k + h][0]), "=r"(q[2 * k + h][1]),
                             "=r"(q[2 * k + h][2]), "=r"(q[2 * k + h][3]) : "r"((src ^ h << 4) + k * 2048));
        }
        if (!mbar_wait_warp(done + before.slot * 8, before.phase)) return;
        const uint32_t dst = dst0 + x.slot * kSlotBytes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t s = e[k] ? e[k] << 7 : 0x40u;        // 2^(e - 127) in bf16 (255: infinity)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t v[8];
                codes_to_bf16(q[2 * k + h], s | s << 16, v);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"((dst ^ (2 * h) << 4) + k * 2048), "r"(v[0]),
                             "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"((dst ^ (2 * h + 1) << 4) + k * 2048), "r"(v[4]),
                             "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
            }
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(filled + x.slot * 8);
            mbar_arrive(raw_empty + raw.slot * 8);
        }
        x.advance(kFillGroups);
        raw.advance(kFillGroups);
        before.advance(kFillGroups);
    }
}

// Four neighbouring elements of dW's row, column k on.
template <typename Args>
__device__ __forceinline__ void store_four(const Args &a, int64_t at, int64_t k, float x0, float x1, float x2, float x3)
{
    if (a.vector && k < a.n_in) {           // n_in is a multiple of 4 and dw aligned to four elements
        if (a.grad_type == NOVAK_TYPE_F32)
            *reinterpret_cast<float4 *>(static_cast<float *>(a.dw) + at) = make_float4(x0, x1, x2, x3);
        else
            *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.dw) + at) = make_uint2(bf16_pair(x0, x1), bf16_pair(x2, x3));
    } else {
        const float x[4] = {x0, x1, x2, x3};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < a.n_in) store_param(a.dw, a.grad_type, at + i, x[i]);
    }
}

// Warps 0 ..: the tile.  A warp has 32 rows (its quarter of the lanes) x 128 columns
// of it in registers and adds to them what the tensor cores have summed of a run.
__device__ __forceinline__ void take_out(const KernelArgs &a, Shared &sh, uint32_t tmem, uint32_t rank, int pair)
{
    const Cut &cut = a.cut;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int quarter = warp % 4, side = warp / 4;
    Walk walk(cut, pair);
    Piece piece;
    uint32_t n = 0;
    bool ok = true;
    while (ok && walk.next(piece)) {
        int tn, tk;
        tile_at(cut, piece.tile, tn, tk);
        const int64_t n0 = static_cast<int64_t>(tn) * kTileN + rank * 128;
        float total[128];
#pragma unroll
        for (int i = 0; i < 128; ++i) total[i] = 0.0f;
        for (int left = piece.count; left > 0; left -= kRun) {
            const uint32_t buf = n & 1;
            ok = mbar_wait_warp(smem_addr(&sh.out_full[buf]), (n >> 1) & 1);
            if (!ok) {
                if (lane == 0) atomicAdd(&g_gave_up, 1u);
                break;
            }
            tcgen05_after_sync();
            const uint32_t src = tmem + buf * 256 + side * 128 + (static_cast<uint32_t>(quarter) * 32 << 16);
#pragma unroll
            for (int c = 0; c < 128; c += 16) {
                float v[16];
                tmem_load16(src + c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) total[c + i] += v[i];
            }
            if (left <= kRun) break;            // the last run's columns stay this warp's for a while
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[buf]), 0));
            ++n;
        }
        // The tile goes out in a loop, not unrolled over the registers it is in: code that runs
        // once per tile comes from far away.  So it goes through tensor memory once more.
        const uint32_t at = tmem + (n & 1) * 256 + side * 128 + (static_cast<uint32_t>(quarter) * 32 << 16);
#pragma unroll
        for (int c = 0; c < 128; c += 16) tmem_store16(at + c, total + c);
        tmem_store_wait();
        const bool partial = !piece.whole || cut.all_partial;
        float4 *dst = reinterpret_cast<float4 *>(a.partial) + (static_cast<int64_t>(piece.slot) * 64 + side * 32) * 256 +
                      rank * 128 + quarter * 32 + lane;
        float *turn = sh.turn[warp];
        const int row = lane / 2, col = lane % 2 * 4;
        const int64_t row0 = n0 + quarter * 32 + row, k0 = static_cast<int64_t>(tk) * kTileK + side * 128 + col;
#pragma unroll 1
        for (int c = 0; c < 128; c += 16) {
            float v[16];
            tmem_load16(at + c, v);
            if (!ok)        // nobody takes this for a result
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(0x7fffffffu);
            if (partial) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    dst[(c / 4 + i) * 256] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            } else {
                // through shared memory: four neighbouring columns of sixteen rows per store
#pragma unroll
                for (int h = 0; h < 16; h += 8) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) turn[lane * kPad + i] = v[h + i];
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 32; i += 16) {
                        const float *src = turn + (row + i) * kPad + col;
                        const int64_t k = k0 + c + h;
                        if (row0 + i < a.n_out) store_four(a, (row0 + i) * a.n_in + k, k, src[0], src[1], src[2], src[3]);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok) break;
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[n & 1]), 0));
        ++n;
    }
}

// Warps kSumWarp, + 1: sums over dy's columns, 64 columns of a warp, from shared
// memory.  The tiles of a tile row share the chunks of rows among them.
__device__ __forceinline__ void sum_dy(const KernelArgs &a, Shared &sh, uint32_t dys, uint32_t rank, int pair)
{
    const Cut &cut = a.cut;
    const int half = threadIdx.x / 32 - kSumWarp, lane = threadIdx.x % 32;
    const int chunk = lane % 8, row0 = lane / 8;        // 8 columns of every fourth row
    Walk walk(cut, pair);
    Piece piece;
    Ring<kDySlots> dy;
    while (walk.next(piece)) {
        int tn, tk;
        tile_at(cut, piece.tile, tn, tk);
        StepPos at(cut, piece.first);
        float s[8] = {}, total[8] = {};
        for (int i = 0; i < piece.count; ++i, at.advance(cut)) {
            if (!mbar_wait_warp(smem_addr(&sh.dy_full[dy.slot]), dy.phase)) return;
            if (at.chunk % cut.tiles_k == tk) {
                const uint32_t src = dys + dy.slot * kSlotBytes + half * kHalf;
#pragma unroll 4
                for (int t = row0; t < kRows; t += 4) {
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(src + t * 128 + ((chunk ^ (t & 7)) << 4)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        s[2 * k] += __uint_as_float(w[k] << 16);
                        s[2 * k + 1] += __uint_as_float(w[k] & 0xffff0000u);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.done[dy.slot]));
            dy.advance();
            if (i % kRun == kRun - 1 || i == piece.count - 1) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    total[k] += s[k];
                    s[k] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            total[k] += __shfl_xor_sync(0xffffffffu, total[k], 8);
            total[k] += __shfl_xor_sync(0xffffffffu, total[k], 16);
        }
        if (lane < 8) {
            float4 *dst = reinterpret_cast<float4 *>(a.sums + static_cast<int64_t>(piece.slot) * 256 + rank * 128 + half * 64 + chunk * 8);
            dst[0] = make_float4(total[0], total[1], total[2], total[3]);
            dst[1] = make_float4(total[4], total[5], total[6], total[7]);
        }
    }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
novak_weight_grad_kernel(const __grid_constant__ KernelArgs a, const __grid_constant__ CUtensorMap map,
                         const __grid_constant__ CUtensorMap codes_map)
{
    extern __shared__ uint8_t raw[];
    const uint32_t dys = (smem_addr(raw) + 1023) & ~1023u, xs = dys + kDySlots * kSlotBytes, raws = xs + kXSlots * kSlotBytes;
    Shared &sh = *reinterpret_cast<Shared *>(raw + (raws - smem_addr(raw)) + kRawSlots * kRawBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x / 2;
    const Cut &cut = a.cut;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kDySlots; ++i) {
            mbar_init(smem_addr(&sh.dy_full[i]), 1);
            mbar_init(smem_addr(&sh.done[i]), a.sums ? 1 + kSumWarps : 1);
        }
        for (int i = 0; i < kXSlots; ++i) {
            mbar_init(smem_addr(&sh.full[i]), kGroupWarps + 1);         // the leading CTA's warps and the other CTA
            mbar_init(smem_addr(&sh.filled[i]), kGroupWarps);
        }
        for (int i = 0; i < kRawSlots; ++i) {
            mbar_init(smem_addr(&sh.raw_full[i]), 2);
            mbar_init(smem_addr(&sh.raw_empty[i]), kGroupWarps);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_addr(&sh.out_full[b]), 1);
            mbar_init(smem_addr(&sh.out_empty[b]), 2 * kOutWarps);
        }
        mbar_init(smem_addr(&sh.drained), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc_pair(smem_addr(&sh.tmem), 512);
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;

    // (every warp of a warpgroup executes the same one of the two)
    if (warp < kOutWarps) registers_up<kOutRegs>();
    else registers_down<kOtherRegs>();

    if (warp < kOutWarps) {
        take_out(a, sh, tmem, rank, pair);
    } else if (warp < kLoadWarp) {
        fill_x(a, sh, xs, raws, rank, pair);
    } else if (warp < kCopyWarp) {
        load_codes(a, &codes_map, sh, raws, rank, pair);
    } else if (warp >= kSumWarp) {
        if (a.sums) sum_dy(a, sh, dys, rank, pair);
    } else {
        Walk walk(cut, pair);
        Piece piece;
        bool ok = true;
        Ring<kDySlots> dy;
        if (warp == kCopyWarp && lane == 0) {
            // ---- dy: 64 rows x 128 columns per step, by tensor copies
            Ring<kDySlots> first_open;          // the oldest step whose copy may not have been waited for by anyone
            int64_t issued = 0;
            while (ok && walk.next(piece)) {
                int tn, tk;
                tile_at(cut, piece.tile, tn, tk);
                const int x = tn * kTileN + static_cast<int>(rank) * 128;
                StepPos at(cut, piece.first);
                for (int i = 0; i < piece.count; ++i) {
                    ok = mbar_wait(smem_addr(&sh.done[dy.slot]), dy.phase ^ 1);
                    if (!ok) break;
                    const uint32_t bar = smem_addr(&sh.dy_full[dy.slot]), dst = dys + dy.slot * kSlotBytes;
                    mbar_expect(bar, 2 * kHalf);
                    tma_load_3d(dst, &map, x, at.chunk * kRows, at.plane, bar);
                    tma_load_3d(dst + kHalf, &map, x + 64, at.chunk * kRows, at.plane, bar);
                    at.advance(cut);
                    dy.advance();
                    if (++issued > kDySlots) first_open.advance();
                }
            }
            // Every commit of the leading CTA has arrived here before this CTA leaves ...
            for (int i = 0; ok && i < kDySlots; ++i) {
                ok = mbar_wait(smem_addr(&sh.done[dy.slot]), dy.phase ^ 1);
                dy.advance();
            }
            // ... and so has every copy, where a wait gave up and nobody took them
            if (!ok)
                for (int64_t i = 0; i < min(issued, static_cast<int64_t>(kDySlots)); ++i, first_open.advance())
                    mbar_wait(smem_addr(&sh.dy_full[first_open.slot]), first_open.phase);
        } else if (warp == kMmaWarp && rank == 1) {
            // ---- the leading CTA's products read this CTA's dy and x too: one arrival there
            // tells of both (an arrival at another CTA takes long: no warp that fills makes one)
            Ring<kXSlots> x;
            const uint32_t lead_full = at_rank(smem_addr(&sh.full[0]), 0);
            while (ok && walk.next(piece))
                for (int i = 0; ok && i < piece.count; ++i) {
                    ok = mbar_wait_warp(smem_addr(&sh.dy_full[dy.slot]), dy.phase) && mbar_wait_warp(smem_addr(&sh.filled[x.slot]), x.phase);
                    if (ok && lane == 0) mbar_arrive_cluster(lead_full + x.slot * 8);
                    __syncwarp();
                    dy.advance();
                    x.advance();
                }
        } else if (warp == kMmaWarp) {
            // ---- the products.  The warp stays together and one lane issues, so that the
            // descriptors are the warp's: formed by a lane on its own they cost more time
            // than the products take.
            uint32_t n = 0;
            constexpr uint32_t idesc = instr_desc(256, 256);
            const uint64_t dy0 = operand_desc(dys, kHalf, 1024), x0 = operand_desc(xs, kHalf, 1024);
            Ring<kXSlots> x;
            while (ok && walk.next(piece)) {
                for (int left = piece.count; ok && left > 0; ++n) {
                    const int run = min(left, kRun);
                    left -= run;
                    const uint32_t buf = n & 1, d = tmem + buf * 256;
                    ok = mbar_wait_warp(smem_addr(&sh.out_empty[buf]), ((n >> 1) & 1) ^ 1);
                    tcgen05_after_sync();
                    for (int i = 0; ok && i < run; ++i) {
                        ok = mbar_wait_warp(smem_addr(&sh.dy_full[dy.slot]), dy.phase) && mbar_wait_warp(smem_addr(&sh.full[x.slot]), x.phase);
                        if (!ok) break;
                        tcgen05_after_sync();
                        const uint64_t dy_at = dy0 + dy.slot * (kSlotBytes >> 4), x_at = x0 + x.slot * (kSlotBytes >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kRows / 16; ++k)
                                mma_pair_bf16(d, dy_at + k * (2048 >> 4), x_at + k * (2048 >> 4), idesc, i > 0 || k > 0);
                            mma_commit_pair(smem_addr(&sh.done[dy.slot]));
                            if (i == run - 1) mma_commit_pair(smem_addr(&sh.out_full[buf]));
                        }
                        __syncwarp();
                        dy.advance();
                        x.advance();
                    }
                }
            }
            if (!ok) {      // products in flight end before their operands and sums go
                if (elect_one()) mma_commit_pair(smem_addr(&sh.drained));
                __syncwarp();
                mbar_wait_warp(smem_addr(&sh.drained), 0);
            }
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    if (warp == 0) tmem_free_pair(tmem, 512);
}

// ---- partial tiles and column sums --------------------------------------------------
struct FinishArgs {
    Cut cut;
    const float *partial, *sums;
    const void *weight, *bias;
    int param_type;
    void *dw, *db;
    int grad_type, vector;
    int64_t n_out, n_in;
    int first_tile, n_tiles;        // to be added up; then tiles_n for db
};

// kFinishRows rows of a tile per CTA, two groups of four columns of one per thread.
constexpr int kFinishRows = 8, kFinishCtas = kTileN / kFinishRows;
__global__ void __launch_bounds__(256) novak_weight_grad_finish_kernel(const __grid_constant__ FinishArgs a)
{
    __shared__ float part[32][kFinishRows + 1], total[kFinishRows];
    __shared__ float turn[kFinishRows][kTileK + 4];
    const Cut &cut = a.cut;
    const int group = blockIdx.x % kFinishCtas, item = blockIdx.x / kFinishCtas;
    const bool for_db = item >= a.n_tiles;
    int tn, tk = 0, slot, n;
    if (for_db) tn = item - a.n_tiles;
    else tile_at(cut, a.first_tile + item, tn, tk);
    const int row = threadIdx.x % kFinishRows, lane = threadIdx.x / kFinishRows;
    const int64_t n0 = static_cast<int64_t>(tn) * kTileN + group * kFinishRows;
    if (n0 >= a.n_out) return;
    if (for_db || a.weight) {
        float s = 0.0f;
        for (int k = lane; k < cut.tiles_k; k += 32) {
            tile_slots(cut, tile_index(cut, tn, k), slot, n);
            for (int i = 0; i < n; ++i) s += a.sums[static_cast<int64_t>(slot + i) * 256 + group * kFinishRows + row];
        }
        part[lane][row] = s;
        __syncthreads();
        if (threadIdx.x < kFinishRows) {
            s = 0.0f;
            for (int i = 0; i < 32; ++i) s += part[i][row];
            total[row] = s;
            if (for_db && n0 + row < a.n_out) store_param(a.db, a.grad_type, n0 + row, s);
        }
        if (for_db) return;
    }
    tile_slots(cut, a.first_tile + item, slot, n);
    if (n == 1 && !cut.all_partial) return;         // stored as it was
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = lane + 32 * j;
        const float4 *src = reinterpret_cast<const float4 *>(a.partial) + (static_cast<int64_t>(slot) * 64 + c) * 256 +
                            group * kFinishRows + row;
        float4 v = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float4 p = src[static_cast<int64_t>(i) * 64 * 256];
            v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
        }
        *reinterpret_cast<float4 *>(&turn[row][4 * c]) = v;
    }
    __syncthreads();
    const int64_t k0 = static_cast<int64_t>(tk) * kTileK;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = threadIdx.x / 64 + 4 * j, c = threadIdx.x % 64 * 4;
        const int64_t k = k0 + c;
        if (n0 + r >= a.n_out || k >= a.n_in) continue;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = turn[r][c + i];
            if (a.weight && k + i < a.n_in)
                x[i] = fmaf(x[i], param_at(a.weight, a.param_type, k + i), param_at(a.bias, a.param_type, k + i) * total[r]);
        }
        store_four(a, (n0 + r) * a.n_in + k, k, x[0], x[1], x[2], x[3]);
    }
}

// ---- host ---------------------------------------------------------------------------
struct Layout {
    int planes;
    bool copied;            // dy goes through the workspace
    int64_t ld;             // elements between rows as the tensor copies see them
    Cut cut;
    size_t planes_bytes, partial_bytes, sums_bytes;
};

constexpr size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

// The workspace holds for a call with or without sums and a layer norm's scale.
Layout layout_for(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in, bool affine)
{
    Layout l{};
    l.planes = type == NOVAK_TYPE_F32 ? 3 : 1;
    l.copied = l.planes > 1 || !wide(dy, type, rows);
    l.ld = l.copied ? (n_out + 7) / 8 * 8 : dy.stride;
    l.planes_bytes = l.copied ? round_up(static_cast<size_t>(l.planes) * rows * l.ld * 2) : 0;
    Cut &c = l.cut;
    c.tiles_n = static_cast<int>((n_out + kTileN - 1) / kTileN);
    c.tiles_k = static_cast<int>((n_in + kTileK - 1) / kTileK);
    c.planes = l.planes;
    c.steps = static_cast<int>(l.planes * ((rows + kRows - 1) / kRows));
    constexpr int kPairs = 74;          // pairs of SMs
    const int tiles = c.tiles_n * c.tiles_k;
    c.pairs = kPairs;
    c.waves = tiles / kPairs;
    c.rest = tiles % kPairs;
    c.rest_pairs = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kPairs, static_cast<int64_t>(c.rest) * c.steps / kMinSteps)));
    c.all_partial = affine;
    // (whole tiles take slots behind the pieces' only where they go through the workspace)
    const size_t n_slots = static_cast<size_t>(c.rest_pairs) + c.rest + (affine ? tiles : 0);
    l.partial_bytes = n_slots * kTileN * kTileK * sizeof(float);
    l.sums_bytes = round_up(static_cast<size_t>(slots(c)) * 256 * sizeof(float));
    return l;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

}  // namespace

size_t weight_grad_bytes(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in, bool affine)
{
    if (rows <= kFewRows) return 0;
    const Layout l = layout_for(dy, type, rows, n_out, n_in, affine);
    return l.planes_bytes + l.partial_bytes + l.sums_bytes;
}

cudaError_t weight_grad_gave_up(unsigned *count, cudaStream_t stream)
{
    cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_gave_up, sizeof *count, 0, cudaMemcpyDeviceToHost, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t stream)
{
    if (a.rows <= kFewRows) {
        const dim3 grid(static_cast<unsigned>((a.n_in + kTile - 1) / kTile),
                        static_cast<unsigned>((a.n_out + kTile - 1) / kTile));
        if (a.type == NOVAK_TYPE_F32) novak_weight_grad_few_kernel<0><<<grid, kPlainThreads, 0, stream>>>(a);
        else novak_weight_grad_few_kernel<1><<<grid, kPlainThreads, 0, stream>>>(a);
        return cudaGetLastError();
    }
    const Layout l = layout_for(a.dy, a.type, a.rows, a.n_out, a.n_in, a.weight != nullptr);
    uint8_t *work = static_cast<uint8_t *>(a.work);
    const __nv_bfloat16 *dy = static_cast<const __nv_bfloat16 *>(a.dy.ptr);
    if (l.copied) {
        __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(work);
        const int grid = static_cast<int>(std::min<int64_t>((a.rows * (l.ld / 8) + 255) / 256, 148 * 32));
        if (a.type == NOVAK_TYPE_F32)
            novak_weight_grad_planes_kernel<0><<<grid, 256, 0, stream>>>(static_cast<const float *>(a.dy.ptr), a.dy.stride,
                                                                         out, l.ld, a.rows, a.n_out);
        else
            novak_weight_grad_planes_kernel<1><<<grid, 256, 0, stream>>>(dy, a.dy.stride, out, l.ld, a.rows, a.n_out);
        dy = out;
    }
    const EncodeTiled encode = encoder();
    if (!encode) return cudaErrorNotSupported;
    CUtensorMap map;
    const int64_t plane = a.rows * l.ld;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.n_out), static_cast<cuuint64_t>(a.rows), static_cast<cuuint64_t>(l.planes)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(l.ld) * 2, static_cast<cuuint64_t>(plane) * 2};
    const cuuint32_t box[3] = {64, kRows, 1}, one[3] = {1, 1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16 *>(dy), dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;

    CUtensorMap codes_map;
    const cuuint64_t cdims[2] = {static_cast<cuuint64_t>(act_pitch(a.n_in)), static_cast<cuuint64_t>(a.rows)};
    const cuuint64_t cstride[1] = {static_cast<cuuint64_t>(act_pitch(a.n_in))};
    const cuuint32_t cbox[2] = {128, kRows};
    if (encode(&codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.codes.codes, cdims, cstride, cbox, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;

    // shared memory beyond 48 KB has to be asked for once on each device
    static std::atomic<uint64_t> asked{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && (device >= 64 || !(asked.load() >> device & 1))) {
        e = cudaFuncSetAttribute(novak_weight_grad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        if (e == cudaSuccess && device < 64) asked.fetch_or(uint64_t(1) << device);
    }
    if (e != cudaSuccess) return e;

    const bool sums = a.db || a.weight;
    const int vector = a.n_in % 4 == 0 && reinterpret_cast<uintptr_t>(a.dw) % (a.grad_type == NOVAK_TYPE_F32 ? 16 : 8) == 0;
    KernelArgs k{l.cut, a.codes, act_pitch(a.n_in), a.dw, a.grad_type, vector, a.rows, a.n_out, a.n_in,
                 reinterpret_cast<float *>(work + l.planes_bytes), nullptr};
    float *sums_at = reinterpret_cast<float *>(work + l.planes_bytes + l.partial_bytes);
    if (sums) k.sums = sums_at;
    const int pairs = l.cut.waves > 0 ? l.cut.pairs : l.cut.rest_pairs;
    novak_weight_grad_kernel<<<2 * pairs, kThreads, kSmemBytes, stream>>>(k, map, codes_map);

    FinishArgs f{l.cut, k.partial, sums_at, a.weight, a.bias, a.param_type, a.dw, a.db, a.grad_type, vector,
                 a.n_out, a.n_in, 0, 0};
    const int tiles = l.cut.tiles_n * l.cut.tiles_k, whole = l.cut.waves * l.cut.pairs;
    f.first_tile = l.cut.all_partial ? 0 : whole;
    f.n_tiles = tiles - f.first_tile;
    const int64_t blocks = static_cast<int64_t>(kFinishCtas) * (f.n_tiles + (a.db ? l.cut.tiles_n : 0));
    if (blocks > 0) novak_weight_grad_finish_kernel<<<static_cast<unsigned>(blocks), 256, 0, stream>>>(f);
    return cudaGetLastError();
}

}  // namespace novak
