// Orthogonalised updates by Newton-Schulz products:
//     X = G / max(|G|, eps), then for each triple (a, b, c): A = X X^T,
//     X <- a X + (b A + c A^2) X  (X^T X and products from the right where X is tall).
//
// Numbers.  The products' operands are fp16 with 11 bits, scaled by powers of two (X by 2^12, A
// by 2^11, B = b A + c A^2 by 2^12: the spectra that the caller's polynomials allow keep them
// below 2^16, and what falls out at the other end is 2^-24 of the scale); sums are fp32.  A step
// multiplies small singular values by a = 3.4 and large ones by about 1, so that what X is
// rounded by, 2^-12 of the LARGE ones, would be a hundred times as much of the small ones five
// steps later (8e-3 of the result for a gradient of low rank, 0.12 for one of rank one; in bf16
// eight times that).  So X is held as the sum of two fp16 parts, 22 bits, and the linear term
// a X takes both; the products, which the large singular values rule, take the first part
// alone.  The diagonals of A and B, where the sums of squares are and which make up most of a
// matrix close to orthogonal, are held in fp32 apart, zeros standing in their places:
//     (A^2)_ij = (A'^2)_ij + (d_i + d_j) A'_ij  (i != j),  (A^2)_ii = (A'^2)_ii + d_i^2,
//     B X = B' X + diag(B) X.
// diag(B) multiplies X's first part like B' does, so that the rounding that B's few large
// directions leave out stays outside; in the last two steps, after which nothing makes it
// large any more, both parts.  All spectra tried then end within 2e-3 of the exact result.
//
// Memory.  Every matrix is kept as panels of 64 columns: the rows of a panel, 128 bytes each,
// lie one behind the other, rows padded to 128 and columns to 64 with zeros.
#include <algorithm>
#include <atomic>
#include <climits>

#include <cuda_fp16.h>

#include "novak_ops.cuh"
#include "novak_tcgen05.cuh"

namespace novak {
namespace {

constexpr float kScaleX = 4096.0f, kScaleA = 2048.0f, kScaleB = 4096.0f, kScaleLow = 2048.0f;   // (the low part: on top of X's)
constexpr int kPanel = 64, kBlock = 128, kThreads = 256;
constexpr int kUnitRows = 128;              // a unit of the first two kernels: so many rows of a panel

// A matrix as the kernels see it.  Panels' places are in rows of 128 bytes from the workspace's start.
struct Item {
    const void *g;
    void *out;                  // bf16; or theta
    float *m;
    int64_t g_stride, out_stride;
    int rows, cols, tall, side; // side: of A and B
    int x[2], low, gram, poly;  // X's first part (taken in turns), second part, A, B
    int x_pitch, s_pitch;       // rows of a panel
    int diag;                   // floats from the diagonals' start: A's, then B's (s_pitch each)
    int unit, units;            // first unit, how many
    int tile[3], tiles[3];      // of each product: the first one (from the product's first), how many
    float step;
};

struct Work {
    __half *panels;
    float *diags;
    Item *items;
    double *partial;            // per unit
    float2 *scale;              // per matrix: G is multiplied by one, then by the other
    unsigned *arrived;          // per matrix: units, of the first kernel
    unsigned *done;             // per matrix: parts of its tiles that are stored
};

struct Control {
    unsigned ticket, failed, left;      // the next tile; whether a wait gave up; CTAs that are through
};

struct Layout {
    int64_t panel_rows = 0, diag_floats = 0, units = 0;
    size_t diags, items, partial, scale, arrived, done, control, bytes;
};

constexpr size_t round_up(size_t n) { return (n + 255) / 256 * 256; }
__host__ __device__ constexpr int pad_to(int64_t n, int to) { return static_cast<int>((n + to - 1) / to * to); }

// Places of one more matrix behind those that are there.
bool place(Layout &l, int64_t rows, int64_t cols, Item &it)
{
    it.rows = static_cast<int>(rows);
    it.cols = static_cast<int>(cols);
    it.tall = rows > cols;
    it.side = static_cast<int>(std::min(rows, cols));
    it.x_pitch = pad_to(rows, kBlock);
    it.s_pitch = pad_to(it.side, kBlock);
    const int64_t x = (cols + kPanel - 1) / kPanel * it.x_pitch, s = static_cast<int64_t>((it.side + kPanel - 1) / kPanel) * it.s_pitch;
    if (l.panel_rows + 3 * x + 2 * s > INT_MAX - (1 << 24)) return false;       // (boxes beyond the last panel have places too)
    int64_t at = l.panel_rows;
    for (int *p : {&it.x[0], &it.x[1], &it.low}) {
        *p = static_cast<int>(at);
        at += x;
    }
    for (int *p : {&it.gram, &it.poly}) {
        *p = static_cast<int>(at);
        at += s;
    }
    l.panel_rows = at;
    it.diag = static_cast<int>(l.diag_floats);
    l.diag_floats += 2 * it.s_pitch;
    it.unit = static_cast<int>(l.units);
    it.units = static_cast<int>(x / kUnitRows);
    l.units += it.units;
    return true;
}

bool finish_layout(Layout &l, int n)
{
    l.diags = static_cast<size_t>(l.panel_rows) * 128;
    l.items = l.diags + round_up(l.diag_floats * sizeof(float));
    l.partial = l.items + round_up(n * sizeof(Item));
    l.scale = l.partial + round_up(l.units * sizeof(double));
    l.arrived = l.scale + round_up(n * sizeof(float2));
    l.done = l.arrived + round_up(n * sizeof(unsigned));
    l.control = l.done + round_up(n * sizeof(unsigned));
    l.bytes = l.control + round_up(sizeof(Control));
    return true;
}

// ---- device: what the kernels share -------------------------------------------------
// The matrix that `unit` belongs to, by the whole warp: of the items' first units the last one
// that is not above it.
__device__ __forceinline__ int item_of(const Item *items, int n, int unit)
{
    int lo = 0, count = n;          // the answer is in [lo, lo + count)
    while (count > 1) {
        const int stride = (count + 31) / 32, at = lo + static_cast<int>(threadIdx.x % 32) * stride;
        const unsigned below = __ballot_sync(0xffffffffu, at < lo + count && items[at].unit <= unit);
        const int k = 31 - __clz(static_cast<int>(below));      // (the first always is)
        const int end = lo + count;
        lo += k * stride;
        count = min(stride, end - lo);
    }
    return lo;
}

struct HostItems {
    static constexpr int kMost = 200;        // (a launch takes 32764 bytes)
    Item item[kMost];
};

__global__ void novak_orthogonalize_items_kernel(const __grid_constant__ HostItems from, int first, int count, Work w, Control *control)
{
    start();
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        w.items[first + i] = from.item[i];
        w.arrived[first + i] = w.done[first + i] = 0;
    }
    if (threadIdx.x == 0) *control = Control{0, 0, 0};
}

struct Momentum {
    int on, nesterov;
    float momentum;
};

// An element of G: of g, or of the momentum that g is part of.
template <int TYPE>
__device__ __forceinline__ float update_of(const Item &it, const Momentum &mo, int64_t row, int64_t col, bool advance)
{
    const float g = param_at(it.g, TYPE, row * it.g_stride + col);
    if (!mo.on) return g;
    float *p = it.m + row * it.cols + col;
    float m = *p;
    if (advance) *p = m = fmaf(mo.momentum, m, g);
    return mo.nesterov ? fmaf(mo.momentum, m, g) : m;
}

// |G|^2 in 64 bits (a square in fp32 would be lost below 1e-19), a sum per unit; the CTA whose
// unit is its matrix's last to arrive adds them up in order.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) novak_orthogonalize_norm_kernel(Work w, int n, Momentum mo, float eps)
{
    __shared__ double sums[kThreads / 32];
    __shared__ bool last;
    start();
    const int which = item_of(w.items, n, blockIdx.x);
    const Item &it = w.items[which];
    const int unit = static_cast<int>(blockIdx.x) - it.unit, blocks = it.x_pitch / kUnitRows;
    const int row0 = unit % blocks * kUnitRows, col0 = unit / blocks * kPanel;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    double sum = 0.0;
    for (int i = warp; i < kUnitRows; i += kThreads / 32)
        for (int k = 0; k < 2; ++k) {
            const int row = row0 + i, col = col0 + 32 * k + lane;
            if (row < it.rows && col < it.cols) {
                const double x = update_of<TYPE>(it, mo, row, col, true);
                sum = fma(x, x, sum);
            }
        }
    const auto reduce = [&](double x) {
        for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        __syncthreads();
        if (lane == 0) sums[warp] = x;
        __syncthreads();
        x = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) x += sums[i];
        return x;
    };
    sum = reduce(sum);
    if (threadIdx.x == 0) {
        w.partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(w.arrived + which, 1u) + 1 == static_cast<unsigned>(it.units);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int i = threadIdx.x; i < it.units; i += kThreads) sum += __ldcg(w.partial + it.unit + i);
    sum = sqrt(reduce(sum));
    // (a norm that is not finite makes everything of the matrix NaN)
    const double scale = !(sum < INFINITY) ? NAN : sum > 0.0 ? kScaleX / fmax(sum, static_cast<double>(eps)) : 0.0;
    const float tiny = scale > 1e36 ? 0x1p100f : 1.0f;          // (its reciprocal is beyond fp32)
    if (threadIdx.x == 0) w.scale[which] = make_float2(tiny, static_cast<float>(scale / tiny));
}

// X's two parts in units of 2^-12: v is close to hi + lo / 2^11.
__device__ __forceinline__ void split(float v, __half &hi, __half &lo)
{
    hi = __float2half_rn(v);
    lo = __float2half_rn((v - __half2float(hi)) * kScaleLow);
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) novak_orthogonalize_start_kernel(Work w, int n, Momentum mo)
{
    start();
    const int which = item_of(w.items, n, blockIdx.x);
    const Item &it = w.items[which];
    const int unit = static_cast<int>(blockIdx.x) - it.unit, blocks = it.x_pitch / kUnitRows;
    const int row0 = unit % blocks * kUnitRows, panel = unit / blocks;
    const float2 scale = w.scale[which];
    for (int e = threadIdx.x; e < kUnitRows * kPanel; e += kThreads) {
        const int row = row0 + e / kPanel, col = panel * kPanel + e % kPanel;
        const float v = row < it.rows && col < it.cols ? update_of<TYPE>(it, mo, row, col, false) * scale.x * scale.y : 0.0f;
        const int64_t at = (static_cast<int64_t>(panel) * it.x_pitch + row) * kPanel + e % kPanel;
        split(v, w.panels[static_cast<int64_t>(it.x[0]) * kPanel + at], w.panels[static_cast<int64_t>(it.low) * kPanel + at]);
    }
}

// ---- the products on the tensor cores --------------------------------------------------
// One launch does all products of all matrices.  A tile is 256 rows by 256 (or 128) columns of one
// product; pairs of SMs (cta_group::2, 128 rows each) take tiles in one fixed order, step by
// step, product by product, matrix by matrix, each pair the next one that nobody has.  A
// product needs all tiles of the one before of ITS matrix: each matrix has a count of the
// parts that are stored, and the warp that brings operands waits for it.  Whatever a tile
// waits for is before it in that order, so that some pair has it already and waits for
// nothing behind it: no matter how many pairs are at work, they come to an end.  Other
// matrices' tiles fill the time in which one's are awaited.
//
// A and B are symmetric: of their 128 x 128 blocks those on and above the diagonal are computed, and
// stored twice, as they are and transposed.  Operands come from the panels as they lie, in 64 x 64
// boxes: a panel's rows are an operand's rows with the summed dimension contiguous (X X^T, A, B),
// or the summed dimension (X^T X, the X of B X) with the operand's other one contiguous.
//
// In each CTA: warps 0-7 take tiles out (a warp a quarter of the lanes, warps 0-3 the left half of
// the columns), warp 8 brings operands, warp 9 issues the products (of the pair: in the
// leading CTA), warp 10 of the leading CTA hands tiles out.
constexpr int kPairs = 74, kStages = 6, kRing = 2;
constexpr int kBoxBytes = kPanel * 128, kStageBytes = 4 * kBoxBytes, kSideBytes = 2 * kBoxBytes;
constexpr int kOutWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kTileWarp = 10, kTcThreads = 384;

// What is to be done for a tile, as the leading CTA's warp 10 writes it into both CTAs.
struct Tile {
    int what;               // 0: A; 1: B; 2: X; -1: no more
    int which, step, columns;
    int row, col;           // of the tile
    int steps;              // of 64 products
    int a, a_step, a_half;  // rows of 128 bytes: the first box of a CTA's 128 rows, the next 64 products, its second box
    int b, b_step, b_half;
    int a_rank, b_rank;     // what the second CTA of the pair adds to a and b
    uint32_t descriptor;    // of the instruction
    unsigned need;          // parts of this matrix that have to be stored before
    int announced;          // 0: a test's tile whose end nobody is told
};
constexpr int kTileWords = sizeof(Tile) / 4;
static_assert(kTileWords <= 32, "a lane each");

struct Shared {
    alignas(8) uint64_t full[kStages], empty[kStages], out_full[2], out_empty[2], tile_full[kRing], tile_empty[kRing], want, drained;
    uint32_t tmem;
    Tile tiles[kRing];
    alignas(16) float columns[2][128];      // a half's columns of a diagonal
};
constexpr int kSmemBytes = kStages * kStageBytes + 2 * kSideBytes + 1024 + static_cast<int>(sizeof(Shared));
static_assert(kSmemBytes <= 227 * 1024, "shared memory");

struct ProductArgs {
    Work w;
    Control *control;
    int n, steps;
    int first[4];               // tiles of a step: where each product's begin, and all
    int columns[3];             // of a tile
    float coefficients[kMostSteps][3];
    float decay;
    int theta;
    int64_t withheld;
    uint64_t wait_ns;
};

__device__ unsigned g_orthogonalize_gave_up;    // waits that ran out, since the library was loaded

__device__ __forceinline__ unsigned load_acquire(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ void gave_up(const ProductArgs &a)
{
    atomicAdd(&g_orthogonalize_gave_up, 1u);
    atomicExch(&a.control->failed, 1u);
}

// Stored parts of a matrix: until there are `need` of them.
__device__ __forceinline__ bool wait_parts(const ProductArgs &a, const unsigned *done, unsigned need)
{
    if (load_acquire(done) >= need) return true;
    uint64_t t0 = 0;
    for (;;) {
        for (int i = 0; i < 64; ++i) {
            if (load_acquire(done) >= need) return true;
            __nanosleep(20);
        }
        if (load_acquire(&a.control->failed)) return false;
        const uint64_t t = global_ns();
        if (t0 == 0) t0 = t;
        else if (t - t0 > a.wait_ns) return false;
    }
}

// Waits for a barrier that the other CTA of the pair completes, with what it wrote before.
__device__ __forceinline__ bool mbar_try_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\n"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n"
                 "selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, uint64_t limit)
{
    uint64_t t0 = 0;
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_cluster(bar, parity)) return true;
        const uint64_t t = global_ns();
        if (t0 == 0) t0 = t;
        else if (t - t0 > limit) return false;
    }
}
__device__ __forceinline__ void mbar_arrive_release(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A 64 x 64 box, whose arrival is told to a barrier of the leading CTA.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, int y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(map), "r"(0), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// The four warps of one half of the columns; whether all of them agree.
__device__ __forceinline__ void half_sync(int side)
{
    asm volatile("bar.sync %0, 128;" ::"r"(1 + side) : "memory");
}
__device__ __forceinline__ bool half_agree(int side, bool yes)
{
    uint32_t all;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\n"
                 "barrier.cta.red.and.aligned.pred q, %2, 128, p;\n"
                 "selp.u32 %0, 1, 0, q;\n}" : "=r"(all) : "r"(static_cast<uint32_t>(yes)), "r"(1 + side) : "memory");
    return all != 0;
}

// fp16 x fp16 -> fp32; `a_across`, `b_across`: the operand's own dimension is the contiguous one.
__device__ constexpr uint32_t fp16_descriptor(int columns, bool a_across, bool b_across)
{
    return 1u << 4 | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) | static_cast<uint32_t>(columns >> 3) << 17 | (256u >> 4) << 24;
}

__device__ __forceinline__ void tmem_load32(uint32_t tmem, float (&v)[32])
{
    tmem_load16(tmem, reinterpret_cast<float (&)[16]>(v[0]));
    tmem_load16(tmem + 16, reinterpret_cast<float (&)[16]>(v[16]));
}

// Tile number t, by the whole warp.
__device__ __forceinline__ Tile tile_at(const ProductArgs &a, int64_t t)
{
    Tile r{};
    const int per_step = a.first[3];
    r.step = static_cast<int>(t / per_step);
    int rest = static_cast<int>(t % per_step);
    r.what = rest >= a.first[2] ? 2 : rest >= a.first[1] ? 1 : 0;
    rest -= a.first[r.what];
    // the matrix: the last one whose tiles begin at `rest` or before
    int lo = 0, count = a.n;
    while (count > 1) {
        const int stride = (count + 31) / 32, at = lo + static_cast<int>(threadIdx.x % 32) * stride, end = lo + count;
        const unsigned below = __ballot_sync(0xffffffffu, at < end && a.w.items[at].tile[r.what] <= rest);
        lo += (31 - __clz(static_cast<int>(below))) * stride;
        count = min(stride, end - lo);
    }
    r.which = lo;
    const Item &it = a.w.items[lo];
    rest -= it.tile[r.what];
    const int n = r.columns = a.columns[r.what], turn = r.step & 1;
    if (r.what < 2) {
        // of row i of tiles those from column 256 i on
        const int across = (it.side + n - 1) / n, skip = 256 / n;
        int i = 0;
        for (int left = across; rest >= left; left -= skip, ++i) rest -= left;
        r.row = 256 * i;
        r.col = (skip * i + rest) * n;
    } else {
        const int across = (it.cols + n - 1) / n;
        r.row = rest / across * 256;
        r.col = rest % across * n;
    }
    const int half = n / 2;
    const auto along = [&](int base, int pitch, int row, int &at, int &step, int &second) {      // summed dimension contiguous
        at = base + row;
        step = pitch;
        second = 64;
    };
    const auto across = [&](int base, int pitch, int col, int &at, int &step, int &second) {     // its own dimension is
        at = base + col / kPanel * pitch;
        step = 64;
        second = pitch;
    };
    const bool x_across = r.what == 0 ? it.tall != 0 : it.tall == 0;
    const int depth = r.what == 0 ? (it.tall ? it.rows : it.cols) : it.side;
    r.steps = (depth + 63) / 64;
    bool a_across = false, b_across = false;
    if (r.what == 0) {
        a_across = b_across = x_across;
        if (x_across) {
            across(it.x[turn], it.x_pitch, r.row, r.a, r.a_step, r.a_half);
            across(it.x[turn], it.x_pitch, r.col, r.b, r.b_step, r.b_half);
        } else {
            along(it.x[turn], it.x_pitch, r.row, r.a, r.a_step, r.a_half);
            along(it.x[turn], it.x_pitch, r.col, r.b, r.b_step, r.b_half);
        }
    } else if (r.what == 1) {
        along(it.gram, it.s_pitch, r.row, r.a, r.a_step, r.a_half);
        along(it.gram, it.s_pitch, r.col, r.b, r.b_step, r.b_half);
    } else if (it.tall) {
        along(it.x[turn], it.x_pitch, r.row, r.a, r.a_step, r.a_half);
        along(it.poly, it.s_pitch, r.col, r.b, r.b_step, r.b_half);
    } else {
        along(it.poly, it.s_pitch, r.row, r.a, r.a_step, r.a_half);
        across(it.x[turn], it.x_pitch, r.col, r.b, r.b_step, r.b_half);
        b_across = true;
    }
    r.a_rank = a_across ? 2 * r.a_half : 128;
    r.b_rank = b_across ? half / kPanel * r.b_half : half;
    r.descriptor = fp16_descriptor(n, a_across, b_across);
    const unsigned s = it.tiles[0], x = it.tiles[2];        // (as many of B as of A unless their tiles differ)
    const unsigned before = r.what == 0 ? 0 : r.what == 1 ? s : s + it.tiles[1];
    r.need = 4u * (static_cast<unsigned>(r.step) * (s + it.tiles[1] + x) + before);
    r.announced = t != a.withheld;
    return r;
}

// ---- taking a tile out
// Packed fp16 (or bf16) pairs of 64 columns of a thread's row: into a half's place in shared
// memory, as the boxes of a panel's rows lie there (128 bytes a row, 16-byte pieces
// changing places by the row's number).
__device__ __forceinline__ void put_row(uint32_t place, int r, const uint32_t (&h)[32])
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place + r * 128 + ((j ^ (r & 7)) << 4)), "r"(h[4 * j]), "r"(h[4 * j + 1]),
                     "r"(h[4 * j + 2]), "r"(h[4 * j + 3]) : "memory");
}
// The same transposed: the columns become rows, the 128 rows two boxes' columns.
__device__ __forceinline__ void put_column(uint32_t place, int r, const uint32_t (&h)[32])
{
    const uint32_t at = place + (r >> 6) * kBoxBytes + (r & 7) * 2;
    const int piece = (r & 63) >> 3;
#pragma unroll
    for (int c = 0; c < 64; ++c)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + c * 128 + ((piece ^ (c & 7)) << 4)),
                     "h"(static_cast<uint16_t>(c & 1 ? h[c / 2] >> 16 : h[c / 2])) : "memory");
}

// Two boxes of a half's place on their way to rows y0 and y1 (-1: not stored).
__device__ __forceinline__ void send(const CUtensorMap *map, uint32_t place, int side, bool issuer, int y0, int y1)
{
    fence_async_shared();
    half_sync(side);
    if (issuer) {
        if (y0 >= 0) store_box(map, y0, place);
        if (y1 >= 0) store_box(map, y1, place + kBoxBytes);
        stores_commit();
    }
}
// The half's place is free again.
__device__ __forceinline__ void reclaim(int side, bool issuer)
{
    if (issuer) stores_read();
    half_sync(side);
}

__device__ __forceinline__ uint32_t pack_half(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// 32 columns of a row of a panel, 64 bytes, past the first-level cache (other SMs wrote it).
__device__ __forceinline__ void get_row(const __half *panels, int64_t row, int half, uint32_t (&h)[16])
{
    const uint4 *p = reinterpret_cast<const uint4 *>(panels + row * kPanel + 32 * half);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 v = __ldcg(p + j);
        h[4 * j] = v.x;
        h[4 * j + 1] = v.y;
        h[4 * j + 2] = v.z;
        h[4 * j + 3] = v.w;
    }
}

// A half's 64 columns (bf16: two to a word; theta's step: fp32, 32 columns at a time) to the caller's
// rows, from shared memory, so that a row's pieces go out together.
template <bool THETA>
__device__ __forceinline__ void write_out(const ProductArgs &a, const Item &it, uint32_t place, int t, int row0, int col0)
{
    constexpr int kEach = THETA ? 4 : 8;            // elements of a piece
    const bool vector = THETA ? it.cols % 4 == 0 && (reinterpret_cast<uintptr_t>(it.out) & 15u) == 0
                              : it.out_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(it.out) & 15u) == 0;
#pragma unroll 2
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + t / 8, j = t % 8, row = row0 + r, col = col0 + j * kEach;
        uint32_t v[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                     : "r"(place + r * 128 + ((j ^ (r & 7)) << 4)) : "memory");
        if (row >= it.rows || col >= it.cols) continue;
        if constexpr (THETA) {
            float *p = static_cast<float *>(it.out) + static_cast<int64_t>(row) * it.out_stride + col;
            if (vector) {
                float4 x = *reinterpret_cast<const float4 *>(p);
                x.x = fmaf(-it.step, __uint_as_float(v[0]), a.decay * x.x);
                x.y = fmaf(-it.step, __uint_as_float(v[1]), a.decay * x.y);
                x.z = fmaf(-it.step, __uint_as_float(v[2]), a.decay * x.z);
                x.w = fmaf(-it.step, __uint_as_float(v[3]), a.decay * x.w);
                *reinterpret_cast<float4 *>(p) = x;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < it.cols) p[k] = fmaf(-it.step, __uint_as_float(v[k]), a.decay * p[k]);
            }
        } else {
            uint16_t *p = static_cast<uint16_t *>(it.out) + static_cast<int64_t>(row) * it.out_stride + col;
            if (vector && col + 8 <= it.cols) {
                *reinterpret_cast<uint4 *>(p) = make_uint4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (col + k < it.cols) p[k] = static_cast<uint16_t>(k & 1 ? v[k / 2] >> 16 : v[k / 2]);
            }
        }
    }
}

// A panel's width of a thread's row (lane of tensor memory), from column `col` on.
__device__ __forceinline__ void take_panel(const ProductArgs &a, const CUtensorMap *map, const Item &it, const Tile &tile, uint32_t src,
                                           uint32_t place, int side, int r, int row0, int col, float *columns)
{
    const bool issuer = r == 0;
    const int row = row0 + r, panel = col / kPanel;
    float *da = a.w.diags + it.diag, *db = da + it.s_pitch;
    if (tile.what < 2) {
        // block row and column of 128
        const int bi = row0 / kBlock, bj = col / kBlock;
        if (bj < bi) return;                // (the same for all of the half)
        const bool mirror = bj > bi;
        const int base = tile.what == 0 ? it.gram : it.poly;
        const float b = a.coefficients[tile.step][1], c = a.coefficients[tile.step][2];
        uint32_t h[32];
        float d_row = 0.0f;
        if (tile.what == 1) {
            if (r < 64) columns[r] = __ldcg(da + col + r);
            d_row = __ldcg(da + row);
        }
        reclaim(side, issuer);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            uint32_t old[16];
            if (tile.what == 1) get_row(a.w.panels, static_cast<int64_t>(it.gram) + static_cast<int64_t>(panel) * it.s_pitch + row, part, old);
            float v[32];
            tmem_load32(src + 32 * part, v);
            const int on = row - col - 32 * part;           // this row's diagonal element is here if in [0, 32)
            if (tile.what == 0) {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if (i == on) {
                        da[row] = v[i] * (1.0f / (kScaleX * kScaleX));
                        v[i] = 0.0f;
                    }
                    v[i] *= kScaleA / (kScaleX * kScaleX);
                }
            } else {
                constexpr float kSquare = 1.0f / (kScaleA * kScaleA);
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float2 pair = unpack_half(old[i / 2]);
                    const float off = (i & 1 ? pair.y : pair.x) * (1.0f / kScaleA), d = d_row + columns[32 * part + i];
                    if (i == on) {
                        db[row] = fmaf(c, fmaf(v[i], kSquare, d_row * d_row), b * d_row);
                        v[i] = 0.0f;
                    } else {
                        v[i] = kScaleB * fmaf(c, fmaf(v[i], kSquare, d * off), b * off);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) h[16 * part + i] = pack_half(v[2 * i], v[2 * i + 1]);
        }
        put_row(place, r, h);
        const int y = base + panel * it.s_pitch + row0;
        send(map, place, side, issuer, y, y + 64);
        if (mirror) {
            reclaim(side, issuer);
            put_column(place, r, h);
            const int z = base + row0 / kPanel * it.s_pitch + col;
            send(map, place, side, issuer, z, row0 + 64 < it.side ? z + it.s_pitch : -1);
        }
        return;
    }
    const bool last = tile.step + 1 == a.steps, full = tile.step + 2 >= a.steps;
    const int turn = tile.step & 1;
    const float ca = a.coefficients[tile.step][0];
    float d_row = 0.0f;
    if (it.tall) {
        if (r < 64) columns[r] = __ldcg(db + col + r);
    } else {
        d_row = __ldcg(db + row);
    }
    reclaim(side, issuer);
    const int64_t at = static_cast<int64_t>(panel) * it.x_pitch + row;
    uint32_t hi[32], lo[32];
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        uint32_t x_hi[16], x_lo[16];
        get_row(a.w.panels, it.x[turn] + at, part, x_hi);
        get_row(a.w.panels, it.low + at, part, x_lo);
        float v[32];
        tmem_load32(src + 32 * part, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 p = unpack_half(x_hi[i]), q = unpack_half(x_lo[i]);
            const float x0 = fmaf(q.x, 1.0f / kScaleLow, p.x), x1 = fmaf(q.y, 1.0f / kScaleLow, p.y);
            const float d0 = it.tall ? columns[32 * part + 2 * i] : d_row, d1 = it.tall ? columns[32 * part + 2 * i + 1] : d_row;
            v[2 * i] = fmaf(v[2 * i], 1.0f / kScaleB, fmaf(d0, full ? x0 : p.x, ca * x0));
            v[2 * i + 1] = fmaf(v[2 * i + 1], 1.0f / kScaleB, fmaf(d1, full ? x1 : p.y, ca * x1));
        }
        if (last) {
            if (a.theta) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place + r * 128 + ((j ^ (r & 7)) << 4)),
                                 "f"(v[4 * j] * (1.0f / kScaleX)), "f"(v[4 * j + 1] * (1.0f / kScaleX)), "f"(v[4 * j + 2] * (1.0f / kScaleX)),
                                 "f"(v[4 * j + 3] * (1.0f / kScaleX)) : "memory");
                half_sync(side);
                write_out<true>(a, it, place, r, row0, col + 32 * part);
                half_sync(side);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) hi[16 * part + i] = bf16_pair(v[2 * i] * (1.0f / kScaleX), v[2 * i + 1] * (1.0f / kScaleX));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                hi[16 * part + i] = pack_half(v[2 * i], v[2 * i + 1]);
                const float2 p = unpack_half(hi[16 * part + i]);
                lo[16 * part + i] = pack_half((v[2 * i] - p.x) * kScaleLow, (v[2 * i + 1] - p.y) * kScaleLow);
            }
        }
    }
    if (!last) {
        const int y = panel * it.x_pitch + row0;
        put_row(place, r, hi);
        send(map, place, side, issuer, it.x[1 - turn] + y, it.x[1 - turn] + y + 64);
        reclaim(side, issuer);
        put_row(place, r, lo);
        send(map, place, side, issuer, it.low + y, it.low + y + 64);
    } else if (!a.theta) {
        put_row(place, r, hi);
        half_sync(side);
        write_out<false>(a, it, place, r, row0, col);
    }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
novak_orthogonalize_products_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ CUtensorMap map)
{
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (smem_addr(raw) + 1023) & ~1023u, places = stages + kStages * kStageBytes;
    Shared &sh = *reinterpret_cast<Shared *>(raw + (places - smem_addr(raw)) + 2 * kSideBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_addr(&sh.full[i]), 1);
            mbar_init(smem_addr(&sh.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&sh.out_full[i]), 1);
            mbar_init(smem_addr(&sh.out_empty[i]), 2 * kOutWarps);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(smem_addr(&sh.tile_full[i]), 1);
            mbar_init(smem_addr(&sh.tile_empty[i]), 2 * kOutWarps + 3);      // who takes, who brings, and who issues
        }
        mbar_init(smem_addr(&sh.want), 1);
        mbar_init(smem_addr(&sh.drained), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc_pair(smem_addr(&sh.tmem), 512);
    if (threadIdx.x == 32 * kLoadWarp) prefetch_map(&map);
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;
    start();

    bool ok = true;
    Ring<kRing> ring;
    // The next tile; its words are this warp's after that, and the place in the ring is given back.
    const auto next = [&](Tile &tile) {
        ok = mbar_wait_cluster(smem_addr(&sh.tile_full[ring.slot]), ring.phase, a.wait_ns);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) {
            if (lane == 0) gave_up(a);
            return false;
        }
        tile = sh.tiles[ring.slot];
        __syncwarp();
        if (lane == 0) mbar_arrive_release(at_rank(smem_addr(&sh.tile_empty[ring.slot]), 0));
        ring.advance();
        return tile.what >= 0;
    };
    Tile tile;
    if (warp < kOutWarps) {
        const int side = warp / 4, r = threadIdx.x % 128;
        const uint32_t place = places + side * kSideBytes, row_of = static_cast<uint32_t>(warp % 4) * 32 << 16;
        float *columns = sh.columns[side];
        uint32_t count = 0;
        for (;;) {
            const uint32_t buf = count & 1;
            bool more = next(tile);
            if (more && !mbar_wait_warp(smem_addr(&sh.out_full[buf]), (count >> 1) & 1, a.wait_ns)) {
                if (lane == 0) gave_up(a);
                ok = false;
            }
            // (where one's wait gave up the others do not go on to barriers that it will not come to)
            ok = half_agree(side, ok);
            if (!ok || !more) break;
            tcgen05_after_sync();
            const Item &it = a.w.items[tile.which];
            const int row0 = tile.row + static_cast<int>(rank) * kBlock, half = tile.columns / 2;
            const int height = tile.what == 2 ? it.x_pitch : it.s_pitch, width = tile.what == 2 ? it.cols : it.side;
            if (row0 < height)
                for (int c = 0; c < half; c += kPanel)
                    if (tile.col + side * half + c < width)
                        take_panel(a, &map, it, tile, tmem + buf * 256 + side * half + c + row_of, place, side, r, row0,
                                   tile.col + side * half + c, columns);
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[buf]), 0));
            ++count;
            // everything of this half is in memory before that is told
            __threadfence();
            half_sync(side);
            if (r == 0 && tile.announced) {
                stores_done();
                asm volatile("fence.proxy.async;" ::: "memory");
                __threadfence();
                asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(a.w.done + tile.which), "r"(1u) : "memory");
            }
        }
        if (r == 0) stores_done();
    } else if (warp == kLoadWarp) {
        Ring<kStages> at;
        int64_t issued = 0;
        const uint32_t full0 = at_rank(smem_addr(&sh.full[0]), 0);
        while (ok && next(tile)) {
            if (lane == 0) {
                ok = wait_parts(a, a.w.done + tile.which, tile.need);
                asm volatile("fence.proxy.async;" ::: "memory");
                const int boxes = tile.columns / 128;
                int ya = tile.a + static_cast<int>(rank) * tile.a_rank, yb = tile.b + static_cast<int>(rank) * tile.b_rank;
                for (int i = 0; ok && i < tile.steps; ++i, ya += tile.a_step, yb += tile.b_step) {
                    ok = mbar_wait(smem_addr(&sh.empty[at.slot]), at.phase ^ 1, a.wait_ns);
                    if (!ok) break;
                    const uint32_t bar = full0 + at.slot * 8, dst = stages + at.slot * kStageBytes;
                    if (rank == 0) mbar_expect(smem_addr(&sh.full[at.slot]), 2 * (2 + boxes) * kBoxBytes);
                    load_box(dst, &map, ya, bar);
                    load_box(dst + kBoxBytes, &map, ya + tile.a_half, bar);
                    load_box(dst + 2 * kBoxBytes, &map, yb, bar);
                    if (boxes == 2) load_box(dst + 3 * kBoxBytes, &map, yb + tile.b_half, bar);
                    at.advance();
                    ++issued;
                    if (rank == 0 && i == max(tile.steps - 3, 0)) mbar_arrive(smem_addr(&sh.want));
                }
                if (!ok) gave_up(a);
            }
            ok = __all_sync(0xffffffffu, ok);
        }
        // every product that reads this CTA's shared memory is over before the CTA leaves
        for (int i = 0; ok && lane == 0 && i < min(issued, static_cast<int64_t>(kStages)); ++i) {
            // (the last kStages uses: the oldest of them is the next slot if all have been used)
            if (issued < kStages && i == 0) at = Ring<kStages>();
            ok = mbar_wait(smem_addr(&sh.empty[at.slot]), issued < kStages ? at.phase : at.phase ^ 1, a.wait_ns);
            at.advance();
        }
        __syncwarp();
        if (rank == 1) mbar_wait_warp(smem_addr(&sh.drained), 0);
    } else if (warp == kMmaWarp && rank == 0) {
        Ring<kStages> at;
        uint32_t count = 0;
        while (ok && next(tile)) {
            const uint32_t buf = count & 1, d = tmem + buf * 256;
            const bool a_across = tile.descriptor >> 15 & 1, b_across = tile.descriptor >> 16 & 1;
            const uint32_t a_next = a_across ? 2048 >> 4 : 32 >> 4, b_next = b_across ? 2048 >> 4 : 32 >> 4;
            const uint64_t a0 = operand_desc(stages, kBoxBytes, 1024), b0 = operand_desc(stages + 2 * kBoxBytes, kBoxBytes, 1024);
            ok = mbar_wait_warp(smem_addr(&sh.out_empty[buf]), ((count >> 1) & 1) ^ 1, a.wait_ns);
            tcgen05_after_sync();
            for (int i = 0; ok && i < tile.steps; ++i) {
                ok = mbar_wait_warp(smem_addr(&sh.full[at.slot]), at.phase, a.wait_ns);
                if (!ok) break;
                tcgen05_after_sync();
                const uint64_t a_at = a0 + at.slot * (kStageBytes >> 4), b_at = b0 + at.slot * (kStageBytes >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_pair_bf16(d, a_at + k * a_next, b_at + k * b_next, tile.descriptor, i > 0 || k > 0);
                    mma_commit_pair(smem_addr(&sh.empty[at.slot]));
                    if (i == tile.steps - 1) mma_commit_pair(smem_addr(&sh.out_full[buf]));
                }
                __syncwarp();
                at.advance();
            }
            if (!ok && lane == 0) gave_up(a);
            ++count;
        }
        if (elect_one()) mma_commit_pair(smem_addr(&sh.drained));
        __syncwarp();
        mbar_wait_warp(smem_addr(&sh.drained), 0);
    } else if (warp == kTileWarp && rank == 0) {
        const int64_t all = static_cast<int64_t>(a.first[3]) * a.steps;
        const uint32_t other = at_rank(smem_addr(&sh.tiles[0]), 1), other_full = at_rank(smem_addr(&sh.tile_full[0]), 1);
        bool more = true;
        // The next tile is taken when this one's last operands are on their way, not before: with fewer
        // tiles than pairs everybody is to have one.
        for (uint32_t taken = 0; more && ok; ++taken) {
            int64_t t = 0;
            if (taken > 0 && !mbar_wait_warp(smem_addr(&sh.want), (taken - 1) & 1, a.wait_ns)) {
                ok = false;
                if (lane == 0) gave_up(a);
            }
            if (lane == 0) t = !ok || load_acquire(&a.control->failed) ? all : atomicAdd(&a.control->ticket, 1u);
            t = __shfl_sync(0xffffffffu, t, 0);
            more = t < all;
            if (more) tile = tile_at(a, t);
            else tile.what = -1;
            if (!__all_sync(0xffffffffu, mbar_wait_cluster(smem_addr(&sh.tile_empty[ring.slot]), ring.phase ^ 1, a.wait_ns))) {
                ok = false;
                if (lane == 0) gave_up(a);
                break;
            }
            if (lane == 0) sh.tiles[ring.slot] = tile;
            __syncwarp();
            if (lane < kTileWords) {
                const uint32_t word = reinterpret_cast<const uint32_t *>(&sh.tiles[ring.slot])[lane];
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(other + ring.slot * static_cast<uint32_t>(sizeof(Tile)) + 4 * lane), "r"(word) : "memory");
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive_release(at_rank(smem_addr(&sh.tile_full[ring.slot]), 0));
                mbar_arrive_release(other_full + ring.slot * 8);
            }
            ring.advance();
        }
    }
    __syncwarp();
    // Where a wait gave up, copies may still be on their way: they are given a moment.
    if (__syncthreads_or(!ok)) {
        const uint64_t t0 = global_ns();
        while (global_ns() - t0 < 2000000) __nanosleep(1000);
    }
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    if (warp == 0) tmem_free_pair(tmem, 512);
    // The last CTA to leave: nobody takes what a failed call left for a result.
    __shared__ bool bad;
    if (threadIdx.x == 0) {
        __threadfence();
        bad = atomicAdd(&a.control->left, 1u) + 1 == gridDim.x && load_acquire(&a.control->failed);
    }
    __syncthreads();
    if (!bad) return;
    for (int i = 0; i < a.n; ++i) {
        const Item &it = a.w.items[i];
        for (int64_t e = threadIdx.x; e < static_cast<int64_t>(it.rows) * it.cols; e += kTcThreads)
            store_param(it.out, a.theta ? NOVAK_TYPE_F32 : NOVAK_TYPE_BF16, e / it.cols * it.out_stride + e % it.cols, __uint_as_float(0x7fffffffu));
    }
}

// Tiles of a product, `columns` wide.
int tiles_of(const Item &it, int what, int columns)
{
    const int rows = what == 2 ? it.rows : it.side, cols = what == 2 ? it.cols : it.side;
    const int down = (rows + 255) / 256, across = (cols + columns - 1) / columns;
    if (what == 2) return down * across;
    int n = 0;
    for (int i = 0; i < down; ++i) n += across - i * (256 / columns);
    return n;
}

}  // namespace

size_t orthogonalize_bytes(const int64_t *rows, const int64_t *cols, int n)
{
    Layout l;
    Item it{};
    int count = 0;
    for (int i = 0; i < n; ++i)
        if (rows[i] > 0 && cols[i] > 0) {
            if (!place(l, rows[i], cols[i], it)) return 0;
            ++count;
        }
    if (count == 0) return 0;
    finish_layout(l, count);
    return l.bytes;
}

cudaError_t orthogonalize_gave_up(unsigned *count, cudaStream_t stream)
{
    cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_orthogonalize_gave_up, sizeof *count, 0, cudaMemcpyDeviceToHost, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

cudaError_t launch_orthogonalize(const OrthArgs &a, cudaStream_t stream)
{
    Layout l;
    Item it{};
    int n = 0, first_of[3] = {};
    int64_t tiles[3][2] = {};           // of a step, by product: of 256 columns, and of 128
    for (int i = 0; i < a.n; ++i)
        if (a.rows[i] > 0 && a.cols[i] > 0) {
            place(l, a.rows[i], a.cols[i], it);
            for (int what = 0; what < 3; ++what)
                for (int narrow = 0; narrow < 2; ++narrow) tiles[what][narrow] += tiles_of(it, what, narrow ? 128 : 256);
            ++n;
        }
    if (n == 0) return cudaSuccess;
    finish_layout(l, n);
    uint8_t *base = static_cast<uint8_t *>(a.work);
    const Work w{reinterpret_cast<__half *>(base), reinterpret_cast<float *>(base + l.diags), reinterpret_cast<Item *>(base + l.items),
                 reinterpret_cast<double *>(base + l.partial), reinterpret_cast<float2 *>(base + l.scale),
                 reinterpret_cast<unsigned *>(base + l.arrived), reinterpret_cast<unsigned *>(base + l.done)};
    ProductArgs p{};
    p.w = w;
    p.control = reinterpret_cast<Control *>(base + l.control);
    p.n = n;
    p.steps = a.steps;
    int64_t most = 0;
    for (int what = 0; what < 3; ++what) {
        const auto waves = [&](int narrow) { return static_cast<double>((tiles[what][narrow] + kPairs - 1) / kPairs); };
        const bool narrow = waves(1) * 0.6 < waves(0);
        p.columns[what] = narrow ? 128 : 256;
        p.first[what + 1] = p.first[what] + static_cast<int>(tiles[what][narrow]);
        most = std::max(most, tiles[what][narrow]);
    }
    Layout again;
    HostItems items;
    int first = 0, count = 0;
    const auto send = [&] {
        const cudaError_t e = launch(novak_orthogonalize_items_kernel, dim3(1), kThreads, 0, stream, items, first, count, w, p.control);
        first += count;
        count = 0;
        return e;
    };
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < a.n && e == cudaSuccess; ++i) {
        if (a.rows[i] == 0 || a.cols[i] == 0) continue;
        place(again, a.rows[i], a.cols[i], it);
        it.g = a.g[i];
        it.out = a.out ? a.out[i] : a.theta[i];
        it.m = a.m ? a.m[i] : nullptr;
        it.g_stride = a.g_stride ? a.g_stride[i] : a.cols[i];
        it.out_stride = a.out ? a.out_stride[i] : a.cols[i];
        it.step = a.step ? static_cast<float>(a.step[i]) : 0.0f;
        for (int what = 0; what < 3; ++what) {
            it.tile[what] = first_of[what];
            it.tiles[what] = tiles_of(it, what, p.columns[what]);
            first_of[what] += it.tiles[what];
        }
        items.item[count++] = it;
        if (count == HostItems::kMost) e = send();
    }
    if (e == cudaSuccess && count > 0) e = send();
    if (e != cudaSuccess) return e;
    const Momentum mo{a.m != nullptr, a.nesterov, a.momentum};
    const dim3 units(static_cast<unsigned>(l.units));
    const bool f32 = a.type == NOVAK_TYPE_F32;
    e = launch(f32 ? novak_orthogonalize_norm_kernel<0> : novak_orthogonalize_norm_kernel<1>, units, kThreads, 0, stream, w, n, mo,
               static_cast<float>(a.eps));
    if (e == cudaSuccess)
        e = launch(f32 ? novak_orthogonalize_start_kernel<0> : novak_orthogonalize_start_kernel<1>, units, kThreads, 0, stream, w, n, mo);
    if (e != cudaSuccess) return e;

    for (int k = 0; k < a.steps; ++k)
        for (int i = 0; i < 3; ++i) p.coefficients[k][i] = a.coefficients[k][i];
    p.decay = a.decay;
    p.theta = a.out == nullptr;
    p.withheld = a.withheld;
    p.wait_ns = a.wait_ns ? a.wait_ns : kWaitNs;
    // the panels as rows of 128 bytes, one behind the other
    const EncodeTiled encode = tensor_map_encoder();
    if (!encode) return cudaErrorNotSupported;
    CUtensorMap map;
    const cuuint64_t dims[2] = {kPanel, static_cast<cuuint64_t>(l.panel_rows)}, strides[1] = {kPanel * 2};
    const cuuint32_t box[2] = {kPanel, kPanel}, one[2] = {1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> asked{0};
    e = ask_shared_memory(novak_orthogonalize_products_kernel, kSmemBytes, asked);
    if (e != cudaSuccess) return e;
    return launch(novak_orthogonalize_products_kernel, dim3(static_cast<unsigned>(2 * std::min<int64_t>(kPairs, most))), kTcThreads, kSmemBytes,
                  stream, p, map);
}

}  // namespace novak
