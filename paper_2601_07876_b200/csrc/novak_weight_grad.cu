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
//   warp 21      the products (of the pair: in the leading CTA).
//
// dy and x both have the summed dimension (rows) outermost, so both operands are
// "M-major" and neither is transposed.
//
// Work: whole tiles as long as every pair gets one; the rows of the tiles that
// are left over are cut evenly over all pairs, partial tiles going to a
// workspace that novak_weight_grad_finish_kernel adds up in a fixed order.
//
// What bounds it (single calls, the same inputs again and again, clocks high; with other
// inputs each time and one call behind the other 16384 x 4096 -> 4096 is 545 us and 12608 x 768 ->
// 2304 with db and a norm 70): 16384 x 4096 -> 4096 bf16 takes 469 us (1173 TFLOP/s), the
// products with every wait but without filling x about 360: a step's 64 rows are 16 KB of dy and 24 KB of codes and x through each SM's shared
// memory besides the 48 KB that the products read, close to what it can deliver.
// 12608 x 768 -> 2304 bf16: 46 us (970 TFLOP/s), of which the partial tiles' way through
// memory takes 5; with db or a layer norm 60, since dy is read once more (sums inside
// this kernel were 75: they take the shared memory's time too).
#include <algorithm>
#include <atomic>

#include "novak_ops.cuh"
#include "novak_tcgen05.cuh"

namespace novak {
namespace {

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

// A layer norm's weight and bias for four columns, k on.
template <typename Args>
__device__ __forceinline__ void load_affine(const Args &a, int64_t k, float (&w)[4], float (&b)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = k + i < a.n_in ? param_at(a.weight, a.param_type, k + i) : 0.0f;
        b[i] = k + i < a.n_in ? param_at(a.bias, a.param_type, k + i) : 0.0f;
    }
}

// ---- little work: the products in fp32 on the ordinary cores ---------------------
constexpr int kTile = 64, kDepth = 32, kPlainThreads = 256;

struct FewArgs : WeightGradArgs {
    int vector;
    unsigned tiles_k;       // (the grid's second dimension would not hold all of n_out's)
};

// A 64 x 64 tile per CTA, 4 x 4 products per thread; 32 rows at a time, the next ones
// on their way while these are worked on.  One launch and no workspace: bound by latency,
// 2.9 us for one row of 1024 -> 1024; 32 x 256 -> 256 3.5 and 1.4 more for every 32 rows.
template <int TYPE>
__global__ void __launch_bounds__(kPlainThreads) novak_weight_grad_few_kernel(FewArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ __align__(16) float sdy[2][kDepth][kTile], sx[2][kDepth][kTile];
    constexpr int kEach = kDepth * kTile / kPlainThreads, kStep = kPlainThreads / kTile;
    const int64_t pitch = (a.n_in + 31) / 32 * 32;
    const unsigned tile_n = blockIdx.x / a.tiles_k, tile_k = blockIdx.x - tile_n * a.tiles_k;
    const int64_t n0 = static_cast<int64_t>(tile_n) * kTile, k0 = static_cast<int64_t>(tile_k) * kTile;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16, rows = static_cast<int>(a.rows);
    // what a thread brings: dy's column n0 + cn of every fourth row; 8 codes of a row
    static_assert(kDepth * kTile / 8 == kPlainThreads, "eight codes each");
    const int cn = threadIdx.x % kTile, rn = threadIdx.x / kTile, rk = threadIdx.x / 8, ck = threadIdx.x % 8 * 8;
    const bool has_n = n0 + cn < a.n_out, has_k = k0 + ck < pitch;
    T y_next[kEach];
    uint2 q_next;
    uint32_t e_next;
    const auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int t = t0 + rn + kStep * i;
            y_next[i] = T(0.0f);
            if (has_n && t < rows) y_next[i] = static_cast<const T *>(a.dy.ptr)[t * a.dy.stride + n0 + cn];
        }
        q_next = make_uint2(0, 0);
        e_next = 0;
        if (has_k && t0 + rk < rows) {
            const int64_t at = (t0 + rk) * pitch + k0 + ck;
            q_next = *reinterpret_cast<const uint2 *>(a.codes.codes + at);
            e_next = a.codes.exps[at >> 5];
        }
    };
    float acc[4][4] = {}, sum[4] = {};
    start();
    fetch(0);
    for (int t0 = 0, buf = 0; t0 < rows; t0 += kDepth, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) sdy[buf][rn + kStep * i][cn] = to_float(y_next[i]);
        float v[8];
        dequantize8(q_next, e_next, v);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<float4 *>(&sx[buf][rk][ck + 4 * i]) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        __syncthreads();        // (and nobody is in the other buffers any more when they are next written)
        if (t0 + kDepth < rows) fetch(t0 + kDepth);
        const int depth = min(kDepth, rows - t0);
#pragma unroll 4
        for (int d = 0; d < depth; ++d) {
            const float4 y4 = *reinterpret_cast<const float4 *>(&sdy[buf][d][ty * 4]);
            const float4 x4 = *reinterpret_cast<const float4 *>(&sx[buf][d][tx * 4]);
            const float y[4] = {y4.x, y4.y, y4.z, y4.w}, x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] += y[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(y[i], x[j], acc[i][j]);
            }
        }
    }
    const int64_t k = k0 + tx * 4;
    float w[4], b[4];
    if (a.weight) load_affine(a, k, w, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + ty * 4 + i;
        if (n >= a.n_out) continue;
        if (a.db && tile_k == 0 && tx == 0) store_param(a.db, a.grad_type, n, sum[i]);
        if (k >= a.n_in) continue;
        float *x = acc[i];
        if (a.weight)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(x[j], w[j], b[j] * sum[i]);
        store_four(a, n * a.n_in + k, k, x[0], x[1], x[2], x[3]);
    }
}

// ---- the work, cut up --------------------------------------------------------------
constexpr int kTileN = 256, kTileK = 256;       // dW rows and columns of a pair
constexpr int kRows = 64;                       // rows of dy and x per step
constexpr int kGroupN = 8;                      // tiles whose x is shared by neighbours in time
constexpr int kMinSteps = 4;                    // steps of a cut tile that are worth a pair's while

struct Cut {
    int tiles_n, tiles_k;
    int planes;
    int steps;              // of a tile: planes x ceil(rows / 64)
    int run;                // steps that the tensor cores add up by themselves
    int pairs;              // that run whole tiles
    int waves;              // whole tiles per pair
    int rest;               // tiles left over, after the first waves * pairs
    int rest_pairs;         // pairs among which their steps are cut:
    int64_t share;          // so many each,
    int extra;              // and one more for the first of them
};

struct Piece {
    int tile;
    int first, count;       // steps
    int slot;               // in the workspace, of a tile left over (used where the piece is not all of it)
    bool whole;
};

// The step of the tiles left over that pair p starts with.
__device__ __forceinline__ int64_t rest_start(const Cut &c, int p) { return c.share * p + min(p, c.extra); }

// The pair that has step i of them, and the tile that it is in.
__device__ __forceinline__ int divide(int64_t a, int64_t b)
{
    if (a <= 0x7fffffff && b <= 0x7fffffff) return static_cast<int>(a) / static_cast<int>(b);
    return static_cast<int>(a / b);
}
__device__ __forceinline__ int rest_pair(const Cut &c, int64_t i)
{
    const int64_t longer = (c.share + 1) * c.extra;
    return i < longer ? divide(i, c.share + 1) : c.extra + divide(i - longer, c.share);
}
__device__ __forceinline__ int rest_tile(const Cut &c, int64_t i) { return divide(i, c.steps); }

__host__ __device__ __forceinline__ int slots(const Cut &c) { return c.rest_pairs + c.rest; }

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
    // all steps of the walk, at its start
    __device__ int steps() const { return static_cast<int>(static_cast<int64_t>(c.waves) * c.steps + end - pos); }
    __device__ bool next(Piece &p)
    {
        if (wave < c.waves) {
            p.tile = wave * c.pairs + pair;
            p.first = 0;
            p.count = c.steps;
            p.slot = 0;
            ++wave;
        } else if (pos < end) {
            const int r = rest_tile(c, pos);
            p.tile = c.waves * c.pairs + r;
            p.first = static_cast<int>(pos - static_cast<int64_t>(r) * c.steps);
            p.count = static_cast<int>(min(static_cast<int64_t>(c.steps - p.first), end - pos));
            p.slot = pair + r;          // one more than the piece before has, or two
            pos += p.count;
        } else {
            return false;
        }
        p.whole = p.count == c.steps;
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

// First slot and number of slots (consecutive) of tile r of those left over; one: the
// tile is whole, and not in the workspace.
__device__ __forceinline__ void tile_slots(const Cut &c, int r, int &slot, int &n)
{
    const int64_t first = static_cast<int64_t>(r) * c.steps;
    const int lo = rest_pair(c, first), hi = rest_pair(c, first + c.steps - 1);
    slot = lo + r;
    n = hi - lo + 1;
}

// ---- one pass over dy before the products ----------------------------------------------
// Sums of dy's columns over a part of the rows, for db and for what a layer norm's offset
// is multiplied with: sums[part][ld] (null: not asked for).  256 columns per CTA, 8 per
// lane, the warps on rows in turn.  Bound by HBM: 50432 x 3072 bf16 55 us (5.6 TB/s);
// 12608 x 2304 13.4 (4.3 TB/s: the start and the end count).
// COPY: dy as the tensor copies need it too, out[planes][rows][out_ld] in bf16, out_ld a
// multiple of 8: a copy of a bf16 matrix whose rows are not 16-byte aligned, or the three
// parts of an fp32 one.  Each part is what is left cut to 8 bits toward zero (so that none
// rounds up to an infinity); an infinity or NaN is in the first part alone.
constexpr int kSumRows = 16;            // rows that a CTA is worth
constexpr int kMostParts = 64;

template <int TYPE, bool ALIGNED, bool COPY>
__global__ void __launch_bounds__(256)
novak_weight_grad_sums_kernel(const typename Elem<TYPE>::T *dy, int64_t stride, float *sums, int64_t ld, int64_t rows,
                              int64_t cols, int64_t rows_per_part, __nv_bfloat16 *out, int64_t out_ld)
{
    __shared__ float part[8][256];
    start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t col = (static_cast<int64_t>(blockIdx.x) * 32 + lane) * 8;
    const int64_t row0 = blockIdx.y * rows_per_part, row1 = min(row0 + rows_per_part, rows);
    const int n = static_cast<int>(max(min(cols - col, int64_t(8)), int64_t(0)));
    const void *end = end_of(dy, stride, rows, cols);
    F2 s[4] = {F2(0.0f), F2(0.0f), F2(0.0f), F2(0.0f)};
    constexpr int kAhead = 4;
    for (int64_t row = row0 + warp; row < row1; row += 8 * kAhead) {
        Fetch<TYPE, ALIGNED> raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            raw[i].zero();
            if (row + 8 * i < row1) raw[i].load(dy + (row + 8 * i) * stride + col, n, dy, end);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            F2 v[4];
            raw[i].eight().get(v);
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = s[k] + v[k];
            if (COPY && n > 0 && row + 8 * i < row1) {
                __nv_bfloat16 *dst = out + (row + 8 * i) * out_ld + col;
                Eight<NOVAK_TYPE_BF16> e;
                if constexpr (TYPE == NOVAK_TYPE_BF16) {
                    e.set(v);
                    e.store(dst);
                } else {
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        F2 cut[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float c[2] = {v[k].lo(), v[k].hi()}, left[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t bits = __float_as_uint(c[h]);
                                const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
                                const float whole = c[h];
                                if (finite) c[h] = __uint_as_float(bits & 0xffff0000u);
                                left[h] = finite ? whole - c[h] : 0.0f;
                            }
                            cut[k] = F2(c[0], c[1]);
                            v[k] = F2(left[0], left[1]);
                        }
                        e.set(cut);
                        e.store(dst + p * rows * out_ld);
                    }
                }
            }
        }
    }
    if (!sums) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        part[warp][lane * 8 + 2 * k] = s[k].lo();
        part[warp][lane * 8 + 2 * k + 1] = s[k].hi();
    }
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += part[i][threadIdx.x];
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (at < cols) sums[blockIdx.y * ld + at] = sum;
}

// The parts added up, in order.
__device__ __forceinline__ float column_sum(const float *sums, int parts, int64_t ld, int64_t n)
{
    float s = 0.0f;
#pragma unroll 16
    for (int i = 0; i < parts; ++i) s += sums[i * ld + n];
    return s;
}

// ---- the kernel ----------------------------------------------------------------------
constexpr int kDySlots = 6, kXSlots = 4, kRawSlots = 4;         // steps of dy, of x, of codes
constexpr int kHalf = 64 * kRows * 2;                   // 64 columns of an operand, bf16
constexpr int kSlotBytes = 2 * kHalf;                   // 128 columns
constexpr int kRawBytes = 128 * kRows;                  // codes of 128 columns
constexpr int kOutWarps = 8, kFillWarps = 8, kFillGroups = 2, kLoadWarps = 4;
constexpr int kGroupWarps = kFillWarps / kFillGroups;   // that fill a step's x; the groups take turns
constexpr int kLoadWarp = kOutWarps + kFillWarps, kCopyWarp = kLoadWarp + kLoadWarps, kMmaWarp = kCopyWarp + 1;
constexpr int kThreads = 32 * (kCopyWarp + 4);          // (a warpgroup has four)
// A barrier's parity tells one phase from the next, not from the one after that: whoever
// waits for a slot's use number k has to know that use k - 1 is over.  The two groups do
// not finish steps in order among each other, so a slot of codes belongs to one group for
// good, and one of x too.
static_assert(kRawSlots % kFillGroups == 0 && kRawSlots % kLoadWarps == 0, "slots of codes change hands");
static_assert(kXSlots % kFillGroups == 0, "slots of x change hands");
// Registers per thread: 80 at launch, 768 x 80 = 61440 = 256 x 160 + 512 x 40.
constexpr int kOutRegs = 160, kOtherRegs = 40;

struct Shared {
    alignas(8) uint64_t dy_full[kDySlots], full[kXSlots], filled[kXSlots], x_done[kXSlots], raw_full[kRawSlots], raw_empty[kRawSlots], out_full[2], out_empty[2],
        drained;
    uint64_t done[kDySlots];
    uint32_t tmem;
    uint32_t exps[kRawSlots][kRows];    // of four blocks
    alignas(16) float4 turn[kOutWarps][32 * 8];     // 32 rows x 32 columns
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
    void *dw, *db;
    int grad_type, vector;
    int64_t rows, n_out, n_in;
    float *partial;                 // [slot][64][256 rows][4 columns] per tile
    const float *sums;              // [parts][sums_ld], with db or a layer norm's weight and bias
    int parts;
    int64_t sums_ld;
    const void *weight, *bias;
    int param_type;
    uint64_t wait_ns;               // after which a wait gives up (waits for copies and products in flight: kWaitNs)
    int withheld;                   // a pair that is never told of its first sum, for a test of that; or -1
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
    const int64_t blocks = (a.n_in + 31) / 32;
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
                if (!mbar_wait_warp(smem_addr(&sh.raw_empty[raw.slot]), raw.phase ^ 1, a.wait_ns)) {
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
    if (any) mbar_wait_warp(smem_addr(&sh.raw_full[last.slot]), last.phase);      // (whoever fills may have given up)
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
    const int steps = Walk(a.cut, pair).steps();
    Ring<kXSlots> x(group);
    Ring<kRawSlots> raw(group);
    const uint32_t done = smem_addr(&sh.x_done[0]), filled = smem_addr(rank == 0 ? &sh.full[0] : &sh.filled[0]);
    const uint32_t raw_full = smem_addr(&sh.raw_full[0]), raw_empty = smem_addr(&sh.raw_empty[0]);
    for (int step = group; step < steps; step += kFillGroups) {
        if (!mbar_wait_warp(raw_full + raw.slot * 8, raw.phase, a.wait_ns)) return;
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
        if (!mbar_wait_warp(done + x.slot * 8, x.phase ^ 1, a.wait_ns)) return;
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
    }
    // every commit of the leading CTA has arrived here before this CTA leaves
    for (int i = 0; i < kXSlots; i += kFillGroups, x.advance(kFillGroups))
        if (!mbar_wait_warp(done + x.slot * 8, x.phase ^ 1, a.wait_ns)) return;
}

// Warps 0 ..: the tile.  A warp has 32 rows (its quarter of the lanes) x 128 columns
// of it in registers and adds to them what the tensor cores have summed of a run.
// Where a wait gave up, NaNs go out in place of this piece and of all that follow it.
__device__ __forceinline__ void take_out(const KernelArgs &a, Shared &sh, uint32_t tmem, uint32_t rank, int pair)
{
    const Cut &cut = a.cut;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int quarter = warp % 4, side = warp / 4;
    Walk walk(cut, pair);
    Piece piece;
    uint32_t n = 0;
    bool ok = true;
    while (walk.next(piece)) {
        int tn, tk;
        tile_at(cut, piece.tile, tn, tk);
        const int64_t n0 = static_cast<int64_t>(tn) * kTileN + rank * 128;
        float total[128];
#pragma unroll
        for (int i = 0; i < 128; ++i) total[i] = 0.0f;
        for (int left = piece.count; ok && left > 0; left -= cut.run) {
            const uint32_t buf = n & 1;
            ok = mbar_wait_warp(smem_addr(&sh.out_full[buf]), (n >> 1) & 1, a.wait_ns);
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
            if (left <= cut.run) break;            // the last run's columns stay this warp's for a while
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[buf]), 0));
            ++n;
        }
        // The tile goes out in a loop, not unrolled over the registers it is in: code that runs
        // once per tile comes from far away.  So it goes through tensor memory once more.
        const uint32_t at = tmem + (n & 1) * 256 + side * 128 + (static_cast<uint32_t>(quarter) * 32 << 16);
#pragma unroll
        for (int c = 0; c < 128; c += 16)
            if (ok) tmem_store16(at + c, total + c);
        tmem_store_wait();
        const bool partial = !piece.whole;
        float4 *dst = reinterpret_cast<float4 *>(a.partial) + (static_cast<int64_t>(piece.slot) * 64 + side * 32) * 256 +
                      rank * 128 + quarter * 32 + lane;
        const uint32_t turn = smem_addr(sh.turn[warp]);
        const int row = lane / 8, col = lane % 8;               // four rows, eight groups of four columns
        const int64_t row0 = n0 + quarter * 32 + row, k0 = static_cast<int64_t>(tk) * kTileK + side * 128 + 4 * col;
        float mine = 0.0f;              // lane i: the column sum of dy for row i
        const bool bias = a.db && tk == 0 && side == 0;
        if ((a.weight || bias) && !partial && n0 + quarter * 32 + lane < a.n_out) {
            mine = column_sum(a.sums, a.parts, a.sums_ld, n0 + quarter * 32 + lane);
            if (bias) store_param(a.db, a.grad_type, n0 + quarter * 32 + lane, mine);
        }
#pragma unroll 1
        for (int c = 0; c < 128; c += 32) {
            float v[32];
            if (ok) {
                tmem_load16(at + c, reinterpret_cast<float (&)[16]>(v[0]));
                tmem_load16(at + c + 16, reinterpret_cast<float (&)[16]>(v[16]));
            } else {        // nobody takes this for a result
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7fffffffu);
            }
            if (partial) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    dst[(c / 4 + i) * 256] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            } else {
                // through shared memory, so that a store has whole lines of 32 columns; a row's
                // groups of four change places by the row's number, which spreads them over all banks
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (lane * 8 + (i ^ (lane & 7))) * 16),
                                 "f"(v[4 * i]), "f"(v[4 * i + 1]), "f"(v[4 * i + 2]), "f"(v[4 * i + 3]) : "memory");
                __syncwarp();
                float w[4], b[4];
                if (a.weight) load_affine(a, k0 + c, w, b);
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    float x[4];
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3])
                                 : "r"(turn + ((row + i) * 8 + (col ^ ((row + i) & 7))) * 16) : "memory");
                    if (a.weight) {
                        const float s = __shfl_sync(0xffffffffu, mine, row + i);
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = fmaf(x[j], w[j], b[j] * s);
                    }
                    if (row0 + i < a.n_out) store_four(a, (row0 + i) * a.n_in + k0 + c, k0 + c, x[0], x[1], x[2], x[3]);
                }
                __syncwarp();
            }
        }
        if (!ok) continue;
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[n & 1]), 0));
        ++n;
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
            mbar_init(smem_addr(&sh.done[i]), 1);
        }
        for (int i = 0; i < kXSlots; ++i) {
            mbar_init(smem_addr(&sh.full[i]), kGroupWarps + 1);         // the leading CTA's warps and the other CTA
            mbar_init(smem_addr(&sh.filled[i]), kGroupWarps);
            mbar_init(smem_addr(&sh.x_done[i]), 1);
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
    if (threadIdx.x == 32 * kCopyWarp) {
        prefetch_map(&map);
        prefetch_map(&codes_map);
    }
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;
    start();

    // (every warp of a warpgroup executes the same one of the two)
    if (warp < kOutWarps) registers_up<kOutRegs>();
    else registers_down<kOtherRegs>();

    if (warp < kOutWarps) {
        take_out(a, sh, tmem, rank, pair);
    } else if (warp < kLoadWarp) {
        fill_x(a, sh, xs, raws, rank, pair);
    } else if (warp < kCopyWarp) {
        load_codes(a, &codes_map, sh, raws, rank, pair);
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
                    ok = mbar_wait(smem_addr(&sh.done[dy.slot]), dy.phase ^ 1, a.wait_ns);
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
                ok = mbar_wait(smem_addr(&sh.done[dy.slot]), dy.phase ^ 1, a.wait_ns);
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
                    ok = mbar_wait_warp(smem_addr(&sh.dy_full[dy.slot]), dy.phase, a.wait_ns) &&
                         mbar_wait_warp(smem_addr(&sh.filled[x.slot]), x.phase, a.wait_ns);
                    if (ok && lane == 0) mbar_arrive_cluster(lead_full + x.slot * 8);
                    __syncwarp();
                    dy.advance();
                    x.advance();
                }
            mbar_wait_warp(smem_addr(&sh.drained), 0);
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
                    const int run = min(left, cut.run);
                    left -= run;
                    const uint32_t buf = n & 1, d = tmem + buf * 256;
                    ok = mbar_wait_warp(smem_addr(&sh.out_empty[buf]), ((n >> 1) & 1) ^ 1, a.wait_ns);
                    tcgen05_after_sync();
                    for (int i = 0; ok && i < run; ++i) {
                        ok = mbar_wait_warp(smem_addr(&sh.dy_full[dy.slot]), dy.phase, a.wait_ns) &&
                             mbar_wait_warp(smem_addr(&sh.full[x.slot]), x.phase, a.wait_ns);
                        if (!ok) break;
                        tcgen05_after_sync();
                        const uint64_t dy_at = dy0 + dy.slot * (kSlotBytes >> 4), x_at = x0 + x.slot * (kSlotBytes >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kRows / 16; ++k)
                                mma_pair_bf16(d, dy_at + k * (2048 >> 4), x_at + k * (2048 >> 4), idesc, i > 0 || k > 0);
                            mma_commit_pair(smem_addr(&sh.x_done[x.slot]));
                            mma_commit_pair(smem_addr(&sh.done[dy.slot]));
                            if (i == run - 1 && (n > 0 || pair != a.withheld)) mma_commit_pair(smem_addr(&sh.out_full[buf]));
                        }
                        __syncwarp();
                        dy.advance();
                        x.advance();
                    }
                }
            }
            // products in flight end, and every commit arrives in both CTAs, before operands, sums and
            // barriers go (whoever would have waited for them may have given up)
            if (elect_one()) mma_commit_pair(smem_addr(&sh.drained));
            __syncwarp();
            mbar_wait_warp(smem_addr(&sh.drained), 0);
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    if (warp == 0) tmem_free_pair(tmem, 512);
}

// ---- partial tiles, db -------------------------------------------------------------------
struct FinishArgs {
    Cut cut;
    const float *partial, *sums;
    int parts;
    int64_t sums_ld;
    const void *weight, *bias;
    int param_type;
    void *dw, *db;
    int grad_type, vector;
    int64_t n_out, n_in;
};

// kFinishRows rows of a tile that was cut per CTA, two groups of four columns of one per
// thread.  The parts are mostly in L2: 27 tiles from 101 parts (26 MB) take 5 us.
constexpr int kFinishRows = 8, kFinishCtas = kTileN / kFinishRows;
__global__ void __launch_bounds__(256) novak_weight_grad_finish_kernel(const __grid_constant__ FinishArgs a)
{
    __shared__ float total[kFinishRows], part[32][kFinishRows + 1];
    __shared__ float turn[kFinishRows][kTileK + 4];
    const Cut &cut = a.cut;
    start();
    const int group = blockIdx.x % kFinishCtas, item = blockIdx.x / kFinishCtas;
    int tn, tk, slot, n;
    tile_at(cut, cut.waves * cut.pairs + item, tn, tk);
    tile_slots(cut, item, slot, n);
    const int64_t n0 = static_cast<int64_t>(tn) * kTileN + group * kFinishRows;
    if (n == 1 || n0 >= a.n_out) return;
    const int row = threadIdx.x % kFinishRows, lane = threadIdx.x / kFinishRows;
    const bool bias = a.db && tk == 0;
    if (a.weight || bias) {
        float s = 0.0f;
        for (int i = lane; i < a.parts; i += 32) s += a.sums[i * a.sums_ld + n0 + row];        // (padded to whole tiles)
        part[lane][row] = s;
    }
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
    if (a.weight || bias) {
        if (threadIdx.x < kFinishRows) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) s += part[i][threadIdx.x];
            total[threadIdx.x] = s;
            if (bias && n0 + row < a.n_out) store_param(a.db, a.grad_type, n0 + row, s);
        }
        __syncthreads();
    }
    const int c = threadIdx.x % 64 * 4;
    const int64_t k = static_cast<int64_t>(tk) * kTileK + c;
    float w[4], b[4];
    if (a.weight) load_affine(a, k, w, b);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = threadIdx.x / 64 + 4 * j;
        if (n0 + r >= a.n_out || k >= a.n_in) continue;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = turn[r][c + i];
            if (a.weight) x[i] = fmaf(x[i], w[i], b[i] * total[r]);
        }
        store_four(a, (n0 + r) * a.n_in + k, k, x[0], x[1], x[2], x[3]);
    }
}

// ---- host ---------------------------------------------------------------------------
struct Layout {
    int planes;
    bool copied;            // dy goes through the workspace
    bool cut_up;            // some tiles do
    int64_t ld;             // elements between rows as the tensor copies see them
    Cut cut;
    int parts;              // of the rows, in sums of dy's columns
    int64_t rows_per_part, sums_ld;
    size_t planes_bytes, partial_bytes, sums_bytes;
};

constexpr size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

// Whether the ordinary cores are done before the tensor cores' kernels are under way
// (us here and there: 64 x 256 -> 256 4.9 and 11.1, 192 x 256 -> 256 10.7 and 12.2, 256 x
// 256 -> 256 13.4 and 12.1; 64 x 1024 -> 1024 7.4 and 11.5, 128 x 1024 -> 1024 12.5 and
// 12.2, 40 x 2048 -> 2048 15.1 and 12.2).  Up to 16 rows it is writing dW that takes time.
bool little(int64_t rows, int64_t n_out, int64_t n_in)
{
    return rows <= 16 || (rows <= 192 && static_cast<double>(rows) * n_out * n_in <= 1e8);
}

// (The workspace is the same with and without db and a layer norm's weight and bias.)
Layout layout_for(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in)
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
    // The tensor cores' sums round toward zero, so that a chain's error grows with its length: it is cut
    // every 1024 rows, and every 256 products of an fp32 dy, from which more is expected (250 rows in one
    // chain: 9.6e-7 off, cut 3.1e-7, an fp32 sum 2.8e-7; no slower)
    c.run = l.planes > 1 ? 4 : 16;
    constexpr int kPairs = 74;          // pairs of SMs
    const int tiles = c.tiles_n * c.tiles_k;
    c.pairs = kPairs;
    c.waves = tiles / kPairs;
    c.rest = tiles % kPairs;
    // The tiles left over: each whole on a pair of its own, or their steps cut evenly over all pairs, which
    // costs one more kernel and the way of the partial tiles through memory, 256 KB each: as much as about
    // four steps, and one for every eight of them (1024 x 256 -> 256: cut 14 us, whole 19; 1024 x 768 -> 768:
    // 15 and 20; 1024 x 2048 -> 1024: 22 and 19).
    const int64_t left = static_cast<int64_t>(c.rest) * c.steps;
    const int cut_pairs = static_cast<int>(std::min<int64_t>(kPairs, left / kMinSteps));
    c.rest_pairs = std::max(c.rest, 1);
    if (cut_pairs > c.rest && c.steps - left / cut_pairs >= 4 + (cut_pairs + c.rest) / 8) c.rest_pairs = cut_pairs;
    c.share = left / c.rest_pairs;
    c.extra = static_cast<int>(left % c.rest_pairs);
    l.cut_up = c.rest_pairs > c.rest && c.rest > 0;
    l.partial_bytes = l.cut_up ? static_cast<size_t>(slots(c)) * kTileN * kTileK * sizeof(float) : 0;
    // the pass over dy: about four CTAs per SM
    const int64_t column_ctas = (n_out + 255) / 256;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(kMostParts, 148 * 4 / column_ctas), rows / kSumRows));
    l.rows_per_part = (rows + want - 1) / want;
    l.parts = static_cast<int>((rows + l.rows_per_part - 1) / l.rows_per_part);
    l.sums_ld = column_ctas * 256;
    l.sums_bytes = round_up(static_cast<size_t>(l.parts) * l.sums_ld * sizeof(float));
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

template <int TYPE, bool ALIGNED>
cudaError_t launch_sums(const WeightGradArgs &a, const Layout &l, float *sums, __nv_bfloat16 *out, cudaStream_t stream)
{
    constexpr bool kAlways = TYPE == NOVAK_TYPE_F32;
    const auto kernel = out ? novak_weight_grad_sums_kernel<TYPE, ALIGNED, true> : novak_weight_grad_sums_kernel<TYPE, ALIGNED, kAlways>;
    return launch(kernel, dim3(static_cast<unsigned>(l.sums_ld / 256), static_cast<unsigned>(l.parts)), 256, 0, stream,
                  static_cast<const typename Elem<TYPE>::T *>(a.dy.ptr), a.dy.stride, sums, l.sums_ld, a.rows, a.n_out,
                  l.rows_per_part, out, l.ld);
}

}  // namespace

int weight_grad_pairs(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in)
{
    if (little(rows, n_out, n_in)) return 0;
    const Cut c = layout_for(dy, type, rows, n_out, n_in).cut;
    return c.waves > 0 ? c.pairs : c.rest_pairs;
}

size_t weight_grad_bytes(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in)
{
    if (little(rows, n_out, n_in)) return 0;
    const Layout l = layout_for(dy, type, rows, n_out, n_in);
    return l.planes_bytes + l.partial_bytes + l.sums_bytes;
}

cudaError_t weight_grad_gave_up(unsigned *count, cudaStream_t stream)
{
    cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_gave_up, sizeof *count, 0, cudaMemcpyDeviceToHost, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t stream)
{
    const int vector = a.n_in % 4 == 0 && reinterpret_cast<uintptr_t>(a.dw) % (a.grad_type == NOVAK_TYPE_F32 ? 16 : 8) == 0;
    if (little(a.rows, a.n_out, a.n_in)) {
        const int64_t tiles_k = (a.n_in + kTile - 1) / kTile, tiles = tiles_k * ((a.n_out + kTile - 1) / kTile);
        const dim3 grid(static_cast<unsigned>(tiles));      // (below 2^31: dW has 4096 elements for each)
        const FewArgs f{a, vector, static_cast<unsigned>(tiles_k)};
        return launch(a.type == NOVAK_TYPE_F32 ? novak_weight_grad_few_kernel<0> : novak_weight_grad_few_kernel<1>, grid,
                      kPlainThreads, 0, stream, f);
    }
    const Layout l = layout_for(a.dy, a.type, a.rows, a.n_out, a.n_in);
    uint8_t *work = static_cast<uint8_t *>(a.work);
    float *sums = reinterpret_cast<float *>(work + l.planes_bytes + l.partial_bytes);
    const __nv_bfloat16 *dy = static_cast<const __nv_bfloat16 *>(a.dy.ptr);
    if (l.copied || a.db || a.weight) {
        __nv_bfloat16 *copy = l.copied ? reinterpret_cast<__nv_bfloat16 *>(work) : nullptr;
        if (!a.db && !a.weight) sums = nullptr;
        const bool aligned = wide(a.dy, a.type, a.rows) && a.n_out % 8 == 0;
        const auto pass = a.type == NOVAK_TYPE_F32 ? (aligned ? launch_sums<0, true> : launch_sums<0, false>)
                                                   : (aligned ? launch_sums<1, true> : launch_sums<1, false>);
        const cudaError_t e = pass(a, l, sums, copy, stream);
        if (e != cudaSuccess) return e;
        if (copy) dy = copy;
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

    float *partial = reinterpret_cast<float *>(work + l.planes_bytes);
    const KernelArgs k{l.cut, a.codes, a.dw, a.db, a.grad_type, vector, a.rows, a.n_out, a.n_in, partial,
                       sums, l.parts, l.sums_ld, a.weight, a.bias, a.param_type, a.wait_ns ? a.wait_ns : kWaitNs, a.withheld};
    const int pairs = l.cut.waves > 0 ? l.cut.pairs : l.cut.rest_pairs;
    e = launch(novak_weight_grad_kernel, 2 * pairs, kThreads, kSmemBytes, stream, k, map, codes_map);
    if (e != cudaSuccess) return e;

    if (!l.cut_up) return cudaSuccess;
    const FinishArgs f{l.cut, partial, sums, l.parts, l.sums_ld, a.weight, a.bias, a.param_type, a.dw, a.db, a.grad_type,
                       vector, a.n_out, a.n_in};
    return launch(novak_weight_grad_finish_kernel, dim3(static_cast<unsigned>(kFinishCtas * l.cut.rest)), 256, 0, stream, f);
}

}  // namespace novak
