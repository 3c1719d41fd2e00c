// Orthogonalised updates by Newton-Schulz products:
//     X = G / max(|G|, eps), then for each triple (a, b, c): A = X X^T,
//     X <- a X + (b A + c A^2) X  (X^T X and products from the right where X is tall).
//
// Numbers.  Where matrices are small every operand is two fp16 parts and every product three (see there); what
// follows is of the larger ones.  The products' operands are fp16 with 11 bits, scaled by powers of two (X by 2^12, A
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
// large any more, both parts.  The result is then off by 1e-4 (low rank) to 9e-4 (all singular values alike) of its norm
// for dense gradients (the last step without the second part: 1.1e-3 for rank one, before 3e-4, and 2 % less time), and by
// up to 1e-2 where a few elements carry the gradient, whose roundings do not average out.
// Whoever asks for it (`fine`) has operands of two parts here too, X, A and B, and three times the products, one behind
// the other into the same sums: first by first parts, first by second, second by first.  Second parts are not scaled then;
// they end at 2^-24 of the first ones' unit, 2^-36 of |X|.  (4096 x 4096 1.2 and 3.5 ms, 12 of 2304 x 768 and 768 x 768 0.64 and
// 1.2; 5e-4 and 3e-5 off.  What is left are the tensor cores' sums, which cut off what fp32 would round.)
//
// Memory.  Every matrix is kept as panels of 64 columns: the rows of a panel, 128 bytes each,
// lie one behind the other, rows padded to 128 and columns to 64 with zeros.
#include <algorithm>
#include <atomic>
#include <climits>
#include <type_traits>

#include <cuda_fp16.h>

#include "novak_ops.cuh"
#include "novak_tcgen05.cuh"

namespace novak {
namespace {

constexpr float kScaleX = 4096.0f, kScaleA = 2048.0f, kScaleB = 4096.0f, kScaleLow = 2048.0f;   // (the low part: on top of X's)
constexpr int kPanel = 64, kBlock = 128, kThreads = 256;
constexpr int kUnitRows = 128;              // a unit of the first two kernels: so many rows of a panel
constexpr int kMostChunks = 4 * kThreads;   // of a matrix

// A matrix as the kernels see it.  Panels' places are in rows of 128 bytes from the workspace's start.
struct Item {
    const void *g;
    void *out;                  // bf16; or theta
    float *m;
    int64_t g_stride, out_stride;
    int rows, cols, tall, side; // side: of A and B
    int x[2], low[2], gram, poly;       // X's first part (taken in turns), second part (one place unless fine), A, B
    int gram_low, poly_low;     // fine: their second parts
    int x_pitch, s_pitch;       // rows of a panel
    int diag;                   // floats from the diagonals' start: A's, then B's (s_pitch each)
    int unit, units;            // of 128 rows of a panel: first one, how many
    int chunk, chunks;          // of units, whose squares are summed together: first one, how many
    int tile[3], tiles[3];      // of each product: the first one (from the product's first), how many
    float step;
};

struct Work {
    __half *panels;
    float *diags;
    Item *items;
    double *partial;            // per chunk
    unsigned *done;             // per matrix: parts of its tiles that are stored
};

struct Control {
    unsigned ticket, failed, left;      // the next tile; whether a wait gave up; CTAs that are through
};

struct Layout {
    int64_t panel_rows = 0, diag_floats = 0, units = 0, chunks = 0;
    size_t diags, items, partial, done, control, bytes;
};

constexpr size_t kLeastBytes = 4096;        // of matrices that need no workspace: a caller's buffer is never empty, and is checked like any other
constexpr size_t round_up(size_t n) { return (n + 255) / 256 * 256; }
__host__ __device__ constexpr int pad_to(int64_t n, int to) { return static_cast<int>((n + to - 1) / to * to); }

// Places of one more matrix behind those that are there.
bool place(Layout &l, int64_t rows, int64_t cols, bool fine, Item &it)
{
    it.rows = static_cast<int>(rows);
    it.cols = static_cast<int>(cols);
    it.tall = rows > cols;
    it.side = static_cast<int>(std::min(rows, cols));
    it.x_pitch = pad_to(rows, kBlock);
    it.s_pitch = pad_to(it.side, kBlock);
    const int64_t x = (cols + kPanel - 1) / kPanel * it.x_pitch, s = static_cast<int64_t>((it.side + kPanel - 1) / kPanel) * it.s_pitch;
    if (l.panel_rows + (fine ? 4 : 3) * x + (fine ? 4 : 2) * s > INT_MAX - (1 << 24)) return false;     // (boxes beyond the last panel have places too)
    int64_t at = l.panel_rows;
    const auto next = [&](int64_t size, bool own = true) {
        const int p = static_cast<int>(at);
        if (own) at += size;
        return p;
    };
    it.x[0] = next(x);
    it.x[1] = next(x);
    it.low[0] = next(x, fine);
    it.low[1] = next(x);
    it.gram = next(s);
    it.poly = next(s);
    it.gram_low = next(s, fine);
    it.poly_low = next(s, fine);
    l.panel_rows = at;
    it.diag = static_cast<int>(l.diag_floats);
    l.diag_floats += 2 * it.s_pitch;
    it.unit = static_cast<int>(l.units);
    it.units = static_cast<int>(x / kUnitRows);
    l.units += it.units;
    it.chunk = static_cast<int>(l.chunks);
    it.chunks = std::min(it.units, kMostChunks);
    l.chunks += it.chunks;
    return true;
}

void finish_layout(Layout &l, int n)
{
    l.diags = static_cast<size_t>(l.panel_rows) * 128;
    l.items = l.diags + round_up(l.diag_floats * sizeof(float));
    l.partial = l.items + round_up(n * sizeof(Item));
    l.done = l.partial + round_up(l.chunks * sizeof(double));
    l.control = l.done + round_up(n * sizeof(unsigned));
    l.bytes = l.control + round_up(sizeof(Control));
}

// ---- device: what the kernels share -------------------------------------------------
__device__ __forceinline__ uint32_t pack_half(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ F2 halves(uint32_t w)
{
    const float2 p = unpack_half(w);
    return F2(p.x, p.y);
}
__device__ __forceinline__ uint32_t pack_half(F2 x) { return pack_half(x.lo(), x.hi()); }

// Of n items the last one whose first(item) is not above `at`, by the whole warp.
template <typename First> __device__ __forceinline__ int item_of(int n, int at, const First &first)
{
    int lo = 0, count = n;          // the answer is in [lo, lo + count)
    while (count > 1) {
        const int stride = (count + 31) / 32, mine = lo + static_cast<int>(threadIdx.x % 32) * stride, end = lo + count;
        const unsigned below = __ballot_sync(0xffffffffu, mine < end && first(mine) <= at);
        lo += (31 - __clz(static_cast<int>(below))) * stride;       // (the first always is)
        count = min(stride, end - lo);
    }
    return lo;
}

// ---- |G|, and X to begin with
constexpr int kMostItems = 200;             // with one launch, which takes 32764 bytes
template <int N> struct HostItems {         // (a launch of 200 takes 10 us, one of 8 three)
    Item item[N];
};
static_assert(sizeof(HostItems<kMostItems>) + 256 <= 32764, "a launch's parameters");

struct Momentum {
    int on, nesterov;
    float momentum;
};

// A unit of G, four neighbouring elements of 8 rows per thread: f(row, column of the panel, elements), zeros beyond
// the matrix.  G is g, or what momentum makes of it (`advance`: and m goes on).
template <int TYPE, typename F>
__device__ __forceinline__ void for_unit(const Item &it, const Momentum &mo, int unit, bool advance, const F &f)
{
    using T = typename Elem<TYPE>::T;
    const int panels = (it.cols + kPanel - 1) / kPanel, row0 = unit / panels * kUnitRows + threadIdx.x / 16, c = threadIdx.x % 16 * 4;
    const int col = unit % panels * kPanel + c;
    const T *g = static_cast<const T *>(it.g) + col;
    const bool vector = (reinterpret_cast<uintptr_t>(it.g) & (4 * sizeof(T) - 1)) == 0 && it.g_stride % 4 == 0 && it.cols % 4 == 0 &&
                        (reinterpret_cast<uintptr_t>(it.m) & 15u) == 0;
    constexpr int kRows = kUnitRows / (kThreads / 16);
    float v[kRows][4] = {}, m[kRows][4];
    if (vector) {               // (all of them on their way before the first is looked at)
        using Raw = typename std::conditional<TYPE == NOVAK_TYPE_F32, float4, uint2>::type;
        Raw x[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int row = row0 + i * (kThreads / 16);
            x[i] = Raw{};
            if (row < it.rows && col < it.cols) x[i] = *reinterpret_cast<const Raw *>(g + row * it.g_stride);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if constexpr (TYPE == NOVAK_TYPE_F32) {
                v[i][0] = x[i].x; v[i][1] = x[i].y; v[i][2] = x[i].z; v[i][3] = x[i].w;
            } else {
                widen(x[i].x).get(v[i][0], v[i][1]);
                widen(x[i].y).get(v[i][2], v[i][3]);
            }
        }
    } else {
        T x[kRows][4];
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = row0 + i * (kThreads / 16);
                x[i][k] = T(0.0f);
                if (row < it.rows && col + k < it.cols) x[i][k] = g[row * it.g_stride + k];
            }
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = to_float(x[i][k]);
    }
    if (mo.on) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int row = row0 + i * (kThreads / 16);
            if (row >= it.rows || col >= it.cols) continue;
            float *p = it.m + static_cast<int64_t>(row) * it.cols + col;
            if (vector) {
                const float4 x = *reinterpret_cast<const float4 *>(p);
                m[i][0] = x.x; m[i][1] = x.y; m[i][2] = x.z; m[i][3] = x.w;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) m[i][k] = col + k < it.cols ? p[k] : 0.0f;
            }
            if (advance) {
#pragma unroll
                for (int k = 0; k < 4; ++k) m[i][k] = fmaf(mo.momentum, m[i][k], v[i][k]);
                if (vector) {
                    *reinterpret_cast<float4 *>(p) = make_float4(m[i][0], m[i][1], m[i][2], m[i][3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (col + k < it.cols) p[k] = m[i][k];
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = mo.nesterov ? fmaf(mo.momentum, m[i][k], v[i][k]) : m[i][k];
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) f(row0 + i * (kThreads / 16), c, v[i]);
}

__device__ __forceinline__ double sum_of_all(double x, double *scratch)
{
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (threadIdx.x % 32 == 0) scratch[threadIdx.x / 32] = x;
    __syncthreads();
    x = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) x += scratch[i];
    return x;
}

// The sum of a chunk's squares, in 64 bits (a square in fp32 would be lost below 1e-19): a thread's 32 in fp32,
// scaled by a power of two to where they lie.  The items come with the launch, from number `first` on,
// and are put down for the kernels behind.
template <int TYPE, int N>
__global__ void __launch_bounds__(kThreads) novak_orthogonalize_norm_kernel(const __grid_constant__ HostItems<N> from, int first, int count, Work w,
                                                                             Control *control, Momentum mo)
{
    __shared__ double scratch[kThreads / 32];
    start();
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i < count; i += kThreads) {
            w.items[first + i] = from.item[i];
            w.done[first + i] = 0;
        }
        if (threadIdx.x == 0) *control = Control{0, 0, 0};
    }
    const int chunk = from.item[0].chunk + static_cast<int>(blockIdx.x);
    const Item &it = from.item[item_of(count, chunk, [&](int i) { return from.item[i].chunk; })];
    const int64_t mine = chunk - it.chunk;
    double sum = 0.0;
    for (int64_t u = mine * it.units / it.chunks; u < (mine + 1) * it.units / it.chunks; ++u) {
        float x[kUnitRows / (kThreads / 16)][4], top = 0.0f;
        int n = 0;
        for_unit<TYPE>(it, mo, static_cast<int>(u), true, [&](int, int, const float (&v)[4]) {
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, fabsf(x[n][k] = v[k]));
            ++n;
        });
        // 2^-e of top = m 2^e, m in [1, 2) (of an infinity, and of what is below the normal numbers, near enough)
        const int e = max(min(static_cast<int>(__float_as_uint(top) >> 23) - 127, 126), -126);
        const float scale = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        F2 s(0.0f);
#pragma unroll
        for (int i = 0; i < kUnitRows / (kThreads / 16); ++i)
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
                const F2 y = F2(x[i][k], x[i][k + 1]) * F2(scale);
                s = fma2(y, y, s);
            }
        sum += scalbn(static_cast<double>(s.lo() + s.hi()), 2 * e);
    }
    sum = sum_of_all(sum, scratch);
    if (threadIdx.x == 0) w.partial[chunk] = sum;
}

// What G is multiplied by for X in units of 2^-12, in two factors: its norm's reciprocal may be beyond fp32.  (A norm that is
// not finite makes everything of the matrix NaN.)
__device__ __forceinline__ void scale_of(double squares, float eps, float &tiny, float &rest)
{
    const double norm = sqrt(squares), scale = !(norm < INFINITY) ? NAN : norm > 0.0 ? kScaleX / fmax(norm, static_cast<double>(eps)) : 0.0;
    tiny = scale > 1e36 ? 0x1p100f : 1.0f;
    rest = static_cast<float>(scale / tiny);
}

// X's two parts in units of 2^-12.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) novak_orthogonalize_start_kernel(Work w, int n, int64_t units, Momentum mo, float eps, float low_scale)
{
    __shared__ double scratch[kThreads / 32];
    start();
    // this CTA's share of all units, matrix by matrix
    int unit = static_cast<int>(blockIdx.x * units / gridDim.x);
    const int end = static_cast<int>((blockIdx.x + 1) * units / gridDim.x);
    if (unit >= end) return;
    for (int which = item_of(n, unit, [&](int i) { return w.items[i].unit; }); unit < end; ++which) {
        const Item it = w.items[which];
        double norm = 0.0;
        for (int i = threadIdx.x; i < it.chunks; i += kThreads) norm += w.partial[it.chunk + i];
        __syncthreads();
        float tiny, rest;
        scale_of(sum_of_all(norm, scratch), eps, tiny, rest);
        const int panels = (it.cols + kPanel - 1) / kPanel;
        for (const int last = min(end, it.unit + it.units); unit < last; ++unit) {
            const int panel = (unit - it.unit) % panels;
            for_unit<TYPE>(it, mo, unit - it.unit, false, [&](int row, int c, const float (&v)[4]) {
                float x[4];
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = v[k] * tiny * rest;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    hi[k] = pack_half(x[2 * k], x[2 * k + 1]);
                    const float2 h = unpack_half(hi[k]);
                    lo[k] = pack_half((x[2 * k] - h.x) * low_scale, (x[2 * k + 1] - h.y) * low_scale);
                }
                const int64_t at = (static_cast<int64_t>(panel) * it.x_pitch + row) * kPanel + c;
                *reinterpret_cast<uint2 *>(w.panels + static_cast<int64_t>(it.x[0]) * kPanel + at) = make_uint2(hi[0], hi[1]);
                *reinterpret_cast<uint2 *>(w.panels + static_cast<int64_t>(it.low[0]) * kPanel + at) = make_uint2(lo[0], lo[1]);
            });
        }
    }
}

// ---- small matrices ------------------------------------------------------------------
// Of up to 64 rows (or columns), or 128 and no more than 512 of the others: one launch, in which a matrix stays in
// the shared memory of one CTA, or of a cluster of eight, each of which has an eighth of the longer dimension.  The
// fifteen products that depend on one another take the kernel below 7 us each, most of it the way through memory; here
// there are two barriers of the cluster a step (64 x 64: 26 us, by the kernel below 90; 33 x 770: 33 and 120; 128 x 256: 76
// and 106).  The products, 128 x 128 at the most, are ordinary matrix instructions on what lies there: tensor memory would
// add its copies to that chain.
// With so few elements there are few roundings to average: with operands of 11 bits the result of a 2 x 2 matrix would
// be up to 1e-2 off.  So X, A and B are two fp16 parts each, first and second, and products are three: first by first, and first
// by second both ways, in sums of their own.  That is what fp32 arithmetic would give (3e-6 on most spectra, 6e-5
// where G is of rank one), and takes 30 % longer (33 x 770: 25 us; 128 x 256, whose registers do not suffice, 55).
// A CTA sums its part of X X^T; each adds up an eighth of all parts and hands that to everybody; B and B X
// everybody forms alone.  Else numbers are as above.
constexpr int kSmallSide = 128, kSmallThreads = 512, kSmallCluster = 8, kAlone = 128;
constexpr int kSmallMost = 232448 - 1024;   // shared memory

struct SmallItem {
    const void *g;
    void *out;
    float *m;
    int64_t g_stride, out_stride;
    int rows, cols;
    float step;
};
template <int N> struct SmallItems {
    SmallItem item[N];
};
struct SmallArgs {
    float coefficients[kMostSteps][3];
    int steps, theta;
    float decay, eps;
    Momentum mo;
};

// Shared memory of a CTA with `width` columns (of X, or of its transpose where it is tall).
struct SmallLayout {
    int side, blocks, width;        // padded to 16 (from 64 on 32); of 16 x 16, on and above the diagonal; padded to 16
    int pitch, x_pitch;             // in elements: an odd number of 16 bytes
    int sum, a, a_low, hi, lo, diag, bytes; // part at 0, later B's second part
    __host__ __device__ SmallLayout(int s, int w)
    {
        side = pad_to(s, s <= 64 ? 16 : 32);
        blocks = side / 16 * (side / 16 + 1) / 2;
        width = pad_to(w, 16);
        pitch = side + 8;
        x_pitch = width + 8;
        const int square = side * pitch * 2, part = blocks * 1024;
        sum = part;                             // (later B's first part; 16 x 16 in fp32 take more than rows of as many in fp16)
        a = sum + part;
        a_low = a + square;
        hi = a_low + square;
        lo = hi + side * x_pitch * 2;
        diag = lo + side * x_pitch * 2;
        bytes = diag + 2 * side * 4;
    }
};

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_matrices_across(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// d (16 x 8) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void multiply(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float4 load_four_at(uint32_t addr)
{
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ void store_four_at(uint32_t addr, float4 x)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w) : "memory");
}
__device__ __forceinline__ void store_double_at(uint32_t addr, double x)
{
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(x) : "memory");
}

// The CTA's elements of G, several per thread on their way at a time: f(row of X, column of the slice, row, column, element).
// X is G, or its transpose where that is tall.
template <int TYPE, typename F>
__device__ __forceinline__ void for_slice(const SmallItem &it, const Momentum &mo, int first, int width, bool advance, const F &f)
{
    using T = typename Elem<TYPE>::T;
    constexpr int kAhead = 8;
    const bool tall = it.rows > it.cols;
    const unsigned side = min(it.rows, it.cols), inner = tall ? side : width, total = side * width;
    const unsigned inverse = inner > 1 ? 0xffffffffu / inner + 1 : 0;       // (total x inner is below 2^32)
    const T *g = static_cast<const T *>(it.g);
    for (unsigned e0 = threadIdx.x; e0 < total; e0 += kAhead * kSmallThreads) {
        T raw[kAhead];
        float m[kAhead];
        int64_t row[kAhead];
        unsigned at[kAhead], in[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const unsigned e = e0 + k * kSmallThreads, outer = inner > 1 ? __umulhi(e, inverse) : e;
            in[k] = e - outer * inner;
            at[k] = outer;
            const int64_t r = row[k] = tall ? first + static_cast<int>(outer) : static_cast<int>(outer), c = tall ? in[k] : first + in[k];
            raw[k] = T(0.0f);
            m[k] = 0.0f;
            if (e < total) {
                raw[k] = g[r * it.g_stride + c];
                if (mo.on) m[k] = it.m[r * it.cols + c];
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (e0 + k * kSmallThreads >= total) continue;
            const int64_t c = tall ? in[k] : first + in[k];
            float v = to_float(raw[k]);
            if (mo.on) {
                if (advance) it.m[row[k] * it.cols + c] = m[k] = fmaf(mo.momentum, m[k], v);
                v = mo.nesterov ? fmaf(mo.momentum, m[k], v) : m[k];
            }
            f(tall ? in[k] : at[k], tall ? at[k] : in[k], row[k], c, v);
        }
    }
}

template <int TYPE, int N, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(kSmallThreads, 1)
novak_orthogonalize_small_kernel(const __grid_constant__ SmallItems<N> from, const __grid_constant__ SmallArgs args)
{
    extern __shared__ __align__(16) uint8_t raw_shared[];
    __shared__ double scratch[kSmallThreads / 32], norms[C];
    constexpr int kWarps = kSmallThreads / 32;
    const SmallItem &it = from.item[blockIdx.x / C];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rank = C > 1 ? static_cast<int>(cluster_rank()) : 0;
    const int s = min(it.rows, it.cols), l = max(it.rows, it.cols);
    const SmallLayout at(s, (l + C - 1) / C);
    const int first = rank * at.width, width = max(min(l - first, at.width), 0), ks = at.side / 16;
    float *const part = reinterpret_cast<float *>(raw_shared), *const sum = reinterpret_cast<float *>(raw_shared + (C > 1 ? at.sum : 0));
    __half *const gram = reinterpret_cast<__half *>(raw_shared + at.a), *const gram_low = reinterpret_cast<__half *>(raw_shared + at.a_low);
    __half *const poly = reinterpret_cast<__half *>(raw_shared + at.sum), *const poly_low = reinterpret_cast<__half *>(raw_shared);
    __half *const hi = reinterpret_cast<__half *>(raw_shared + at.hi), *const lo = reinterpret_cast<__half *>(raw_shared + at.lo);
    float *const diag_a = reinterpret_cast<float *>(raw_shared + at.diag), *const diag_b = diag_a + at.side;
    const uint32_t gram0 = smem_addr(gram), poly0 = smem_addr(poly), hi0 = smem_addr(hi), gram_low0 = smem_addr(gram_low),
                   poly_low0 = smem_addr(poly_low), lo0 = smem_addr(lo);
    const auto everybody = [] {
        if constexpr (C > 1) cluster_sync();
        else __syncthreads();
    };
    // hi and lo lie one behind the other
    for (int i = threadIdx.x; i < 2 * at.side * at.x_pitch * 2 / 16; i += kSmallThreads) reinterpret_cast<uint4 *>(hi)[i] = make_uint4(0, 0, 0, 0);
    everybody();
    start();

    // ---- |G|, in 64 bits (a square in fp32 would be lost below 1e-19), and X
    double squares = 0.0;
    for_slice<TYPE>(it, args.mo, first, width, true, [&](int, int, int64_t, int64_t, float v) { squares = fma(static_cast<double>(v), static_cast<double>(v), squares); });
    for (int d = 16; d > 0; d >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, d);
    if (lane == 0) scratch[warp] = squares;
    __syncthreads();
    if (threadIdx.x < C) {
        squares = 0.0;
        for (int i = 0; i < kWarps; ++i) squares += scratch[i];
        if constexpr (C > 1) store_double_at(at_rank(smem_addr(&norms[rank]), threadIdx.x), squares);
        else norms[0] = squares;
    }
    everybody();
    double norm = 0.0;
    for (int i = 0; i < C; ++i) norm += norms[i];
    float tiny, rest;
    scale_of(norm, args.eps, tiny, rest);
    for_slice<TYPE>(it, args.mo, first, width, false, [&](int i, int j, int64_t, int64_t, float v) {
        const float x = v * tiny * rest;
        const __half h = __float2half_rn(x);
        hi[i * at.x_pitch + j] = h;
        lo[i * at.x_pitch + j] = __float2half_rn((x - __half2float(h)) * kScaleLow);
    });
    __syncthreads();

    // where a lane's row of a 16 x 16 block begins, for one whose rows are the operand's, and for one whose columns are
    const int row_a = lane % 16, col_a = lane / 16 * 8, row_b = lane / 16 * 8 + lane % 8, col_b = lane / 8 % 2 * 8;
    const auto block_of = [&](int b, int &bi, int &bj) {
        bi = 0;
        for (; b >= ks - bi; ++bi) b -= ks - bi;
        bj = bi + b;
    };
    // the products of rows of a matrix with rows (16 x 16 of them), `low` where its second part is
    const auto rows_by_rows = [&](uint32_t from, uint32_t low, int pitch, int bi, int bj, int steps, float (&d)[2][4]) {
        const uint32_t a0 = ((bi * 16 + row_a) * pitch + col_a) * 2, b0 = ((bj * 16 + row_b) * pitch + col_b) * 2;
        float e[2][4] = {};
        const auto some = [&](auto count, int k) {
            constexpr int kCount = decltype(count)::value;
            uint32_t x[kCount][4], y[kCount][4], x_low[kCount][4], y_low[kCount][4];
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                load_matrices(x[i], from + a0 + (k + i) * 32);
                load_matrices(y[i], from + b0 + (k + i) * 32);
                load_matrices(x_low[i], low + a0 + (k + i) * 32);
                load_matrices(y_low[i], low + b0 + (k + i) * 32);
            }
#pragma unroll
            for (int i = 0; i < kCount; ++i)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    multiply(d[n], x[i], y[i][2 * n], y[i][2 * n + 1]);
                    multiply(e[n], x[i], y_low[i][2 * n], y_low[i][2 * n + 1]);
                    multiply(e[n], x_low[i], y[i][2 * n], y[i][2 * n + 1]);
                }
        };
        int k = 0;
        for (; k + 2 <= steps; k += 2) some(std::integral_constant<int, 2>(), k);
        if (k < steps) some(std::integral_constant<int, 1>(), k);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[n][i] = fmaf(e[n][i], 1.0f / kScaleLow, d[n][i]);
    };
    for (int step = 0; step < args.steps; ++step) {
        const float ca = args.coefficients[step][0], cb = args.coefficients[step][1], cc = args.coefficients[step][2];
        // this CTA's part of X X^T
        for (int b = warp; b < at.blocks; b += kWarps) {
            int bi, bj;
            block_of(b, bi, bj);
            float d[2][4] = {};
            rows_by_rows(hi0, lo0, at.x_pitch, bi, bj, at.width / 16, d);
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2 *>(part + b * 256 + (lane / 4 + 8 * h) * 16 + n * 8 + lane % 4 * 2) = make_float2(d[n][2 * h], d[n][2 * h + 1]);
        }
        everybody();
        if constexpr (C > 1) {
            const int all = at.blocks * 64, each = (all + C - 1) / C;
            for (int i = rank * each + threadIdx.x; i < min((rank + 1) * each, all); i += kSmallThreads) {
                const uint32_t mine = smem_addr(part) + i * 16, there = smem_addr(sum) + i * 16;
                float4 x[C];
#pragma unroll
                for (int r = 0; r < C; ++r) x[r] = load_four_at(at_rank(mine, r));
#pragma unroll
                for (int r = 1; r < C; ++r) x[0] = make_float4(x[0].x + x[r].x, x[0].y + x[r].y, x[0].z + x[r].z, x[0].w + x[r].w);
#pragma unroll
                for (int r = 0; r < C; ++r) store_four_at(at_rank(there, r), x[0]);
            }
            cluster_sync();
        }
        for (int b = warp; b < at.blocks; b += kWarps) {
            int bi, bj;
            block_of(b, bi, bj);
            float there[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) there[k] = sum[b * 256 + k * 32 + lane];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = bi * 16 + 2 * k + lane / 16, j = bj * 16 + lane % 16;
                const float x = there[k] * (1.0f / (kScaleX * kScaleX));
                const float y = i == j ? 0.0f : x * kScaleA;
                const __half h = __float2half_rn(y), low = __float2half_rn((y - __half2float(h)) * kScaleLow);
                if (i == j) diag_a[i] = x;
                gram[i * at.pitch + j] = h;
                gram_low[i * at.pitch + j] = low;
                if (bi != bj) {
                    gram[j * at.pitch + i] = h;
                    gram_low[j * at.pitch + i] = low;
                }
            }
        }
        __syncthreads();
        // B = b A + c A^2
        for (int b = warp; b < at.blocks; b += kWarps) {
            int bi, bj;
            block_of(b, bi, bj);
            float d[2][4] = {};
            rows_by_rows(gram0, gram_low0, at.pitch, bi, bj, ks, d);
            constexpr float kSquare = 1.0f / (kScaleA * kScaleA);
            // two neighbouring columns at a time
            float2 of_a[2][2], di;
            float dj[2][2];
            di = make_float2(diag_a[bi * 16 + lane / 4], diag_a[bi * 16 + lane / 4 + 8]);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int j = bj * 16 + n * 8 + lane % 4 * 2;
                dj[n][0] = diag_a[j];
                dj[n][1] = diag_a[j + 1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int e = (bi * 16 + lane / 4 + 8 * h) * at.pitch + j;
                    const float2 x = unpack_half(*reinterpret_cast<const uint32_t *>(gram + e)), low = unpack_half(*reinterpret_cast<const uint32_t *>(gram_low + e));
                    of_a[n][h] = make_float2(fmaf(low.x, 1.0f / kScaleLow, x.x), fmaf(low.y, 1.0f / kScaleLow, x.y));
                }
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int i = bi * 16 + lane / 4 + 8 * h, j = bj * 16 + n * 8 + lane % 4 * 2;
                    const float mine = h ? di.y : di.x;
                    float v[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        v[k] = fmaf(d[n][2 * h + k], kScaleB * cc * kSquare,
                                    fmaf(cc, mine + dj[n][k], cb) * (kScaleB / kScaleA) * (k ? of_a[n][h].y : of_a[n][h].x));
                        if (i == j + k) {
                            diag_b[i] = fmaf(cc, fmaf(d[n][2 * h + k], kSquare, mine * mine), cb * mine);
                            v[k] = 0.0f;
                        }
                    }
                    const uint32_t w = pack_half(v[0], v[1]);
                    const float2 first_part = unpack_half(w);
                    const uint32_t low = pack_half((v[0] - first_part.x) * kScaleLow, (v[1] - first_part.y) * kScaleLow);
                    const auto put = [&](__half *to, uint32_t x) {
                        *reinterpret_cast<uint32_t *>(to + i * at.pitch + j) = x;
                        if (bi != bj) {
                            to[j * at.pitch + i] = __ushort_as_half(static_cast<uint16_t>(x));
                            to[(j + 1) * at.pitch + i] = __ushort_as_half(static_cast<uint16_t>(x >> 16));
                        }
                    };
                    put(poly, w);
                    put(poly_low, low);
                }
        }
        __syncthreads();
        // X <- a X + B X, 16 columns by one warp, or where there are few by several, each some of the rows: nobody writes before
        // all of them have the columns in registers, or (more than 64 rows, for which these do not suffice) their results
        const auto update = [&](auto rows) {
            constexpr int kRows = decltype(rows)::value;            // times 16
            constexpr int kHeld = kRows <= 4 ? kRows : 0, kResults = kRows <= 4 ? 1 : C > 1 ? 2 : 4;
            const int columns = at.width / 16, helpers = max(min(kWarps / columns, kRows), 1), together = kWarps / helpers;
            for (int c0 = 0; c0 < columns; c0 += together) {
                const int c = c0 + warp / helpers;
                const bool mine = warp / helpers < together && c < columns;
                uint32_t x[kHeld + 1][4], x_low[kHeld + 1][4], w[kResults][2][2], w_low[kResults][2][2];
                const uint32_t x0 = ((lane / 8 % 2 * 8 + lane % 8) * at.x_pitch + c * 16 + lane / 16 * 8) * 2;
                const auto load = [&](int k, int to) {
                    load_matrices_across(x[to], hi0 + x0 + k * 32 * at.x_pitch);
                    load_matrices_across(x_low[to], lo0 + x0 + k * 32 * at.x_pitch);
                };
                const auto everything_is_read = [&] {
                    if (helpers > 1) __syncthreads();
                    else __syncwarp();
                };
                const auto place_of = [&](int m, int n, int h) { return (m * 16 + lane / 4 + 8 * h) * at.x_pitch + c * 16 + lane % 4 * 2 + 8 * n; };
                const auto multiply_rows = [&](int m, uint32_t (&w)[2][2], uint32_t (&w_low)[2][2]) {
                    float d[2][4] = {}, e[2][4] = {};
                    const uint32_t a0 = ((m * 16 + row_a) * at.pitch + col_a) * 2;
                    constexpr int kAhead = kHeld > 0 ? 2 : 1;
#pragma unroll
                    for (int k0 = 0; k0 < kRows; k0 += kAhead) {
                        uint32_t y[kAhead][4], y_low[kAhead][4];
#pragma unroll
                        for (int k = k0; k < k0 + kAhead && k < kRows; ++k) {
                            load_matrices(y[k - k0], poly0 + a0 + k * 32);
                            load_matrices(y_low[k - k0], poly_low0 + a0 + k * 32);
                        }
                        if (kHeld == 0) load(k0, 0);
#pragma unroll
                        for (int k = k0; k < k0 + kAhead && k < kRows; ++k)
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                const uint32_t (&of_x)[4] = x[kHeld > 0 ? k : 0], (&of_x_low)[4] = x_low[kHeld > 0 ? k : 0];
                                multiply(d[n], y[k - k0], of_x[2 * n], of_x[2 * n + 1]);
                                multiply(e[n], y[k - k0], of_x_low[2 * n], of_x_low[2 * n + 1]);
                                multiply(e[n], y_low[k - k0], of_x[2 * n], of_x[2 * n + 1]);
                            }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float db = diag_b[m * 16 + lane / 4 + 8 * h];
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const uint32_t of_hi = *reinterpret_cast<const uint32_t *>(hi + place_of(m, n, h)),
                                           of_lo = *reinterpret_cast<const uint32_t *>(lo + place_of(m, n, h));
                            const F2 both = fma2(halves(of_lo), F2(1.0f / kScaleLow), halves(of_hi));
                            const F2 sum = fma2(F2(e[n][2 * h], e[n][2 * h + 1]), F2(1.0f / kScaleLow), F2(d[n][2 * h], d[n][2 * h + 1]));
                            const F2 v = fma2(sum, F2(1.0f / kScaleB), fma2(F2(db), both, both * F2(ca)));
                            w[n][h] = pack_half(v);
                            w_low[n][h] = pack_half(fma2(halves(w[n][h]), F2(-1.0f), v) * F2(kScaleLow));
                        }
                    }
                };
                const auto put = [&](int m, const uint32_t (&w)[2][2], const uint32_t (&w_low)[2][2]) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            *reinterpret_cast<uint32_t *>(hi + place_of(m, n, h)) = w[n][h];
                            *reinterpret_cast<uint32_t *>(lo + place_of(m, n, h)) = w_low[n][h];
                        }
                };
                if constexpr (kHeld > 0) {
#pragma unroll
                    for (int k = 0; k < kRows; ++k)
                        if (mine) load(k, k);
                    everything_is_read();
                    for (int m = warp % helpers; mine && m < kRows; m += helpers) {
                        multiply_rows(m, w[0], w_low[0]);
                        put(m, w[0], w_low[0]);
                    }
                } else {
                    // (64 columns: four helpers at least; one CTA alone 128: two)
#pragma unroll
                    for (int i = 0; i < kResults; ++i)
                        if (mine && warp % helpers + i * helpers < kRows) multiply_rows(warp % helpers + i * helpers, w[i], w_low[i]);
                    everything_is_read();
#pragma unroll
                    for (int i = 0; i < kResults; ++i)
                        if (mine && warp % helpers + i * helpers < kRows) put(warp % helpers + i * helpers, w[i], w_low[i]);
                }
            }
        };
        switch (ks) {
        case 1: update(std::integral_constant<int, 1>()); break;
        case 2: update(std::integral_constant<int, 2>()); break;
        case 3: update(std::integral_constant<int, 3>()); break;
        case 4: update(std::integral_constant<int, 4>()); break;
        case 6: update(std::integral_constant<int, 6>()); break;
        default: update(std::integral_constant<int, 8>()); break;
        }
        __syncthreads();
    }

    // ---- the result
    const bool tall = it.rows > it.cols;
    const unsigned inner = tall ? s : width, total = static_cast<unsigned>(s) * width;
    const unsigned inverse = inner > 1 ? 0xffffffffu / inner + 1 : 0;
#pragma unroll 4
    for (unsigned e = threadIdx.x; e < total; e += kSmallThreads) {
        const unsigned outer = inner > 1 ? __umulhi(e, inverse) : e, in = e - outer * inner, i = tall ? in : outer, j = tall ? outer : in;
        const int64_t row = tall ? first + j : i, col = tall ? i : first + j;
        const float x = fmaf(__half2float(lo[i * at.x_pitch + j]), 1.0f / kScaleLow, __half2float(hi[i * at.x_pitch + j])) * (1.0f / kScaleX);
        if (args.theta) {
            float *p = static_cast<float *>(it.out) + row * it.out_stride + col;
            *p = fmaf(-it.step, x, args.decay * *p);
        } else {
            static_cast<__nv_bfloat16 *>(it.out)[row * it.out_stride + col] = __float2bfloat16_rn(x);
        }
    }
}

// CTAs of a matrix; 0: it is not small.
int small_ctas(int64_t rows, int64_t cols)
{
    const int64_t s = std::min(rows, cols), l = std::max(rows, cols);
    if (s > kSmallSide || (s > 64 && l > 512)) return 0;
    const auto fits = [&](int ctas) { return SmallLayout(static_cast<int>(s), static_cast<int>((l + ctas - 1) / ctas)).bytes <= kSmallMost; };
    // (64 x 128 alone 24 us; with eight CTAs each has a sixteenth of the work and two barriers a step: 256 columns 24 us)
    return l <= kAlone && fits(1) ? 1 : fits(kSmallCluster) ? kSmallCluster : 0;
}

template <int TYPE, int N, int C>
cudaError_t send_small(const SmallItem *items, int count, const SmallArgs &args, int bytes, cudaStream_t stream)
{
    static std::atomic<uint64_t> asked{0};
    const cudaError_t e = ask_shared_memory(novak_orthogonalize_small_kernel<TYPE, N, C>, kSmallMost, asked);
    if (e != cudaSuccess) return e;
    SmallItems<N> from{};
    std::copy_n(items, count, from.item);
    return launch(novak_orthogonalize_small_kernel<TYPE, N, C>, dim3(static_cast<unsigned>(count * C)), kSmallThreads, bytes, stream, from, args);
}

// All small ones of a call.
template <int TYPE, int C> cudaError_t launch_small(const OrthArgs &a, const SmallArgs &args, cudaStream_t stream)
{
    SmallItem items[kMostItems];
    int count = 0, bytes = 0;
    const auto send = [&] {
        const cudaError_t e = count <= 8 ? send_small<TYPE, 8, C>(items, count, args, bytes, stream) : send_small<TYPE, kMostItems, C>(items, count, args, bytes, stream);
        count = bytes = 0;
        return e;
    };
    for (int i = 0; i < a.n; ++i) {
        if (a.rows[i] == 0 || a.cols[i] == 0 || small_ctas(a.rows[i], a.cols[i]) != C) continue;
        const int s = static_cast<int>(std::min(a.rows[i], a.cols[i])), l = static_cast<int>(std::max(a.rows[i], a.cols[i]));
        bytes = std::max(bytes, SmallLayout(s, (l + C - 1) / C).bytes);
        items[count++] = SmallItem{a.g[i], a.out ? a.out[i] : a.theta[i], a.m ? a.m[i] : nullptr, a.g_stride ? a.g_stride[i] : a.cols[i],
                                   a.out ? a.out_stride[i] : a.cols[i], static_cast<int>(a.rows[i]), static_cast<int>(a.cols[i]),
                                   a.step ? static_cast<float>(a.step[i]) : 0.0f};
        if (count < kMostItems) continue;
        const cudaError_t e = send();
        if (e != cudaSuccess) return e;
    }
    return count > 0 ? send() : cudaSuccess;
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
// In each CTA: warps 0-15 take tiles out (a warp a quarter of the lanes and of the columns, each on
// its own), warp 16 brings operands, warp 17 issues the products (of the pair: in the leading
// CTA), warp 18 of the leading CTA hands tiles out.
constexpr int kPairs = 74, kStages = 5, kRing = 4;
constexpr int kBoxBytes = kPanel * 128, kStageBytes = 4 * kBoxBytes;
constexpr int kPartBytes = 32 * 64, kPlaceBytes = 2 * kPartBytes;       // 32 x 32 elements in fp16; two of those
constexpr int kTold = 32;       // parts of a tile that are told of when they are stored: each warp's that takes it out
constexpr int kOutWarps = 16, kLoadWarp = kOutWarps, kMmaWarp = kLoadWarp + 1, kTileWarp = kMmaWarp + 1, kTcThreads = 32 * (kTileWarp + 1);

// What is to be done for a tile, as the leading CTA's warp 18 sends it to both CTAs: all that they need to know (what
// the matrices' records say comes from L2 each time, since every wait for other SMs' tiles empties the
// first-level cache).
struct Tile {
    int what;               // 0: A; 1: B; 2: X; -1: no more
    int which, step, columns;
    int row, col;           // of the tile
    int steps;              // of 64 products (fine: three times as many)
    int a, a_step, a_half;  // rows of 128 bytes: the first box of a CTA's 128 rows, the next 64 products, its second box
    int b, b_step, b_half;
    int a_rank, b_rank;     // what the second CTA of the pair adds to a and b
    int a_low, b_low;       // fine: from the operands' first parts to their second ones
    uint32_t descriptor;    // of the instruction
    unsigned need;          // parts of this matrix that have to be stored before
    int announced;          // 0: a test's tile whose end nobody is told
    // of what takes it out, in rows of 128 bytes as above:
    int height, width;      // rows and columns that are stored
    int pitch;              // rows of a panel
    int in, low, out, out_low;      // what the tile needs beside its products and its second part, where it goes and where that does
    int diag;               // floats to the diagonal that is needed, or that A's and B's own diagonals are put to
    int tall;
};
constexpr int kTileWords = sizeof(Tile) / 4;
__device__ __forceinline__ uint32_t tile_word(const Tile &t, int i) { return reinterpret_cast<const uint32_t *>(&t)[i]; }
static_assert(kTileWords <= 32, "a lane each");

struct Shared {
    alignas(8) uint64_t full[kStages], empty[kStages], out_full[2], out_empty[2], tile_full[kRing], tile_empty[kRing], ready[kRing], want, drained;
    uint64_t part_full[kOutWarps];
    uint32_t tmem;
    Tile tiles[kRing];
};
constexpr int kSmemBytes = kStages * kStageBytes + kOutWarps * kPlaceBytes + 1024 + static_cast<int>(sizeof(Shared));
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

// Words of a tile into a CTA of the pair, whose barrier there is told of them as of a copy: who waits for
// it needs no fence beyond its CTA (a wait with one of the cluster's took 2000 cycles).
__device__ __forceinline__ void mbar_expect_at(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void send_word(uint32_t dst, uint32_t word, uint32_t bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(dst), "r"(word), "r"(bar) : "memory");
}
// (A tile's words have been used when its place is given back; a release at the cluster's scope would wait for
// all stores on their way, 9000 cycles.)
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Whether a phase is complete, without waiting.
__device__ __forceinline__ bool mbar_try_now(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// A 64 x 64 box, whose arrival is told to a barrier of the leading CTA.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(bar) : "memory");
}
// 32 rows of 32 columns of a panel, in shared memory as 32 rows of 64 bytes whose 16-byte pieces change places by the
// row's number; loads are told to a barrier of this CTA.
__device__ __forceinline__ void load_part(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) { tma_load_2d(dst, map, x, y, bar); }
__device__ __forceinline__ void store_part(const CUtensorMap *map, int x, int y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// fp16 x fp16 -> fp32; `a_across`, `b_across`: the operand's own dimension is the contiguous one.
__device__ constexpr uint32_t fp16_descriptor(int columns, bool a_across, bool b_across)
{
    return 1u << 4 | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) | static_cast<uint32_t>(columns >> 3) << 17 | (256u >> 4) << 24;
}

// Tile number t, by the whole warp.
template <bool FINE> __device__ __forceinline__ Tile tile_at(const ProductArgs &a, int64_t t)
{
    Tile r{};
    const int per_step = a.first[3];
    r.step = static_cast<int>(t / per_step);
    int rest = static_cast<int>(t % per_step);
    r.what = rest >= a.first[2] ? 2 : rest >= a.first[1] ? 1 : 0;
    rest -= a.first[r.what];
    const int lo = item_of(a.n, rest, [&](int i) { return a.w.items[i].tile[r.what]; });
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
    r.need = static_cast<unsigned>(kTold) * (static_cast<unsigned>(r.step) * (s + it.tiles[1] + x) + before);
    r.announced = t != a.withheld;
    r.height = r.what == 2 ? it.x_pitch : it.s_pitch;
    r.width = r.what == 2 ? it.cols : it.side;
    r.pitch = r.height;
    r.in = r.what == 2 ? it.x[turn] : it.gram;
    r.low = r.what == 2 ? it.low[turn] : it.gram_low;
    r.out = r.what == 0 ? it.gram : r.what == 1 ? it.poly : it.x[1 - turn];
    r.out_low = r.what == 0 ? it.gram_low : r.what == 1 ? it.poly_low : it.low[1 - turn];
    if constexpr (FINE) {
        const int of_x = it.low[turn] - it.x[turn], of_poly = it.poly_low - it.poly;
        r.a_low = r.what == 0 ? of_x : r.what == 1 ? it.gram_low - it.gram : it.tall ? of_x : of_poly;
        r.b_low = r.what < 2 ? r.a_low : it.tall ? of_poly : of_x;
    }
    r.diag = it.diag + (r.what == 2 ? it.s_pitch : 0);
    r.tall = it.tall;
    return r;
}

// ---- taking a tile out
// A warp has 32 rows (a thread a lane of tensor memory) and 32 columns at a time.  What it needs of
// X or A comes into shared memory by tensor copies, the results take its place and go from there by
// tensor copies: rows straight from and to memory are 32 lines at a time, of each of which the
// first-level cache moves a sector (15000 cycles a tile of X).  Two places by turns: the next part
// is on its way while one is worked on.
__device__ __forceinline__ uint32_t piece_at(uint32_t place, int row, int piece) { return place + row * 64 + ((piece ^ (row >> 1 & 3)) << 4); }
__device__ __forceinline__ void get_row(uint32_t place, int row, uint32_t (&h)[16])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(h[4 * j]), "=r"(h[4 * j + 1]), "=r"(h[4 * j + 2]), "=r"(h[4 * j + 3])
                     : "r"(piece_at(place, row, j)) : "memory");
}
__device__ __forceinline__ void put_row(uint32_t place, int row, const uint32_t (&h)[16])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece_at(place, row, j)), "r"(h[4 * j]), "r"(h[4 * j + 1]), "r"(h[4 * j + 2]),
                     "r"(h[4 * j + 3]) : "memory");
}
// The same transposed.  Neighbouring lanes exchange halves, so that each has two columns of every other row.
__device__ __forceinline__ void put_across(uint32_t place, const uint32_t (&h)[16])
{
    const int lane = threadIdx.x & 31, odd = lane & 1;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, h[i], 1);
        const uint32_t w = odd ? __byte_perm(other, h[i], 0x7632) : __byte_perm(h[i], other, 0x5410);
        const int row = 2 * i + odd;
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(piece_at(place, row, lane >> 3) + (lane & 6) * 2), "r"(w) : "memory");
    }
}

// The warp's 32 x 32 elements of X to the caller's rows, by way of shared memory, so that rows go out together.
__device__ __forceinline__ void write_out(const Item &it, uint32_t place, int row0, int col, const float (&v)[32])
{
    const int lane = threadIdx.x & 31;
    uint32_t h[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) h[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    put_row(place, lane, h);
    __syncwarp();
    uint16_t *out = static_cast<uint16_t *>(it.out) + row0 * it.out_stride + col;
    if ((reinterpret_cast<uintptr_t>(out) & 15u) == 0 && it.out_stride % 8 == 0 && col + 32 <= it.cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + lane / 4, piece = lane % 4;
            uint4 x;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(piece_at(place, row, piece)) : "memory");
            if (row0 + row < it.rows) *reinterpret_cast<uint4 *>(out + row * it.out_stride + piece * 8) = x;
        }
    } else {
#pragma unroll 4
        for (int row = 0; row < 32; ++row) {
            uint16_t x;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(piece_at(place, row, lane / 8) + lane % 8 * 2) : "memory");
            if (row0 + row < it.rows && col + lane < it.cols) out[row * it.out_stride + lane] = x;
        }
    }
    __syncwarp();
}
// The same for theta's step: fp32, rows of 128 bytes in both of a place's parts.
__device__ __forceinline__ void step_theta(const Item &it, float decay, uint32_t place, int row0, int col, const float (&v)[32])
{
    const int lane = threadIdx.x & 31;
    const auto at = [&](int row, int piece) { return place + row * 128 + ((piece ^ (row & 7)) << 4); };
#pragma unroll
    for (int j = 0; j < 8; ++j)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at(lane, j)), "f"(v[4 * j]), "f"(v[4 * j + 1]), "f"(v[4 * j + 2]), "f"(v[4 * j + 3]) : "memory");
    __syncwarp();
    float *out = static_cast<float *>(it.out) + row0 * it.out_stride + col;
    if ((reinterpret_cast<uintptr_t>(out) & 15u) == 0 && it.out_stride % 4 == 0 && col + 32 <= it.cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 4 + lane / 8, piece = lane % 8;
            float4 x;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at(row, piece)) : "memory");
            if (row0 + row >= it.rows) continue;
            float4 *p = reinterpret_cast<float4 *>(out + row * it.out_stride + piece * 4);
            const float4 t = *p;
            *p = make_float4(fmaf(-it.step, x.x, decay * t.x), fmaf(-it.step, x.y, decay * t.y), fmaf(-it.step, x.z, decay * t.z), fmaf(-it.step, x.w, decay * t.w));
        }
    } else {
#pragma unroll 4
        for (int row = 0; row < 32; ++row) {
            float x;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at(row, lane / 4) + lane % 4 * 4) : "memory");
            if (row0 + row >= it.rows || col + lane >= it.cols) continue;
            float *p = out + row * it.out_stride + lane;
            *p = fmaf(-it.step, x, decay * *p);
        }
    }
    __syncwarp();
}

// A warp that takes tiles out: its place in shared memory and the barrier of what comes there.
template <bool FINE> struct Taking {
    static constexpr float kLow = FINE ? 1.0f : kScaleLow;
    const ProductArgs &a;
    const CUtensorMap *map;
    uint32_t place, bar;
    uint32_t phase;                 // of the barrier
    bool untold;                    // stores are on their way that nobody has been told of
    int told_which, told;           // whose; whether they are to be
    bool own_stores;                // and not by tensor copies alone
    // of a tile:
    int row0, col, parts;           // the warp's first row and column; times 32 columns
    float column, next_column;      // of a diagonal, this lane's, for the part that is worked on and for the next

    // Panels are stored to their ends, which are summed over as zeros; blocks of A and B below the
    // diagonal are not stored from here.  (The same for all of a warp.)
    __device__ __forceinline__ bool here(const Tile &tile, int part) const
    {
        const int c = col + 32 * part, panel = c / kPanel * kPanel;
        return part < parts && panel < tile.width && (tile.what == 2 || c / kBlock >= row0 / kBlock);
    }
    // What a part needs on its way, once what was in its place is out.
    __device__ __forceinline__ void fetch(const Tile &tile, int part)
    {
        if (!here(tile, part)) return;
        const int lane = threadIdx.x & 31, c = col + 32 * part;
        if (tile.what == 1 || (tile.what == 2 && tile.tall)) next_column = __ldcg(a.w.diags + tile.diag + c + lane);
        if (lane == 0) {
            stores_read();
            if (tile.what > 0) {
                const int y = c / kPanel * tile.pitch + row0;
                const bool low = FINE || tile.what == 2;
                mbar_expect(bar, low ? 2 * kPartBytes : kPartBytes);
                load_part(place, map, c % kPanel, tile.in + y, bar);
                if (low) load_part(place + kPartBytes, map, c % kPanel, tile.low + y, bar);
            }
        }
        __syncwarp();
    }
    // Everything of the tile before is in memory, for tensor copies too: told.
    __device__ __forceinline__ void tell()
    {
        if (!untold) return;
        untold = false;
        if (own_stores) __threadfence();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            stores_done();
            if (told) asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(a.w.done + told_which), "r"(1u) : "memory");
        }
        __syncwarp();
    }
    // The diagonal's elements of columns i and i + 1 of a part.
    __device__ __forceinline__ F2 columns(int i) const { return F2(__shfl_sync(0xffffffffu, column, i), __shfl_sync(0xffffffffu, column, i + 1)); }
    // Two elements as they are kept: first part, and second.
    __device__ __forceinline__ void keep(F2 v, uint32_t &h, uint32_t &low) const
    {
        h = pack_half(v);
        if constexpr (FINE) low = pack_half(fma2(halves(h), F2(-1.0f), v));
    }
    // Sixteen columns of A or B, from the sums in tensor memory (and of what A has there: h, and fine low).
    __device__ __forceinline__ void square16(const Tile &tile, int row, bool diagonal, float d_row, const float (&raw)[16],
                                             uint32_t *h, uint32_t *low, int first) const
    {
        const int on = (threadIdx.x & 31) - first;              // this row's diagonal element
        if (tile.what == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) keep(F2(raw[2 * i], raw[2 * i + 1]) * F2(kScaleA / (kScaleX * kScaleX)), h[i], low[i]);
            if (diagonal && on >= 0 && on < 16) {
                float mine = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i == on) mine = raw[i];
                a.w.diags[tile.diag + row] = mine * (1.0f / (kScaleX * kScaleX));
            }
        } else {
            const float cb = a.coefficients[tile.step][1], cc = a.coefficients[tile.step][2];
            constexpr float kSquare = 1.0f / (kScaleA * kScaleA);
            // B' scale = scale (c (square + d a) + b a), a the element of A': (c d + b) a scale + square c scale
            const F2 rest(kScaleB * cc * kSquare), cd(cc * (kScaleB / kScaleA)), bd(fmaf(cc, d_row, cb) * (kScaleB / kScaleA));
            if (diagonal && on >= 0 && on < 16) {
                float mine = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i == on) mine = raw[i];
                a.w.diags[tile.diag + tile.pitch + row] = fmaf(cc, fmaf(mine, kSquare, d_row * d_row), cb * d_row);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const F2 d = columns(first + 2 * i);
                F2 of_a = halves(h[i]);
                if constexpr (FINE) of_a = of_a + halves(low[i]);
                keep(fma2(F2(raw[2 * i], raw[2 * i + 1]), rest, fma2(d, cd, bd) * of_a), h[i], low[i]);
            }
        }
        if (diagonal) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t mask = 2 * i == on ? 0xffff0000u : 2 * i + 1 == on ? 0xffffu : ~0u;
                h[i] &= mask;
                if constexpr (FINE) low[i] &= mask;
            }
        }
    }
    // false: a wait gave up.
    __device__ __forceinline__ bool take(const Tile &tile, uint32_t src)
    {
        const int lane = threadIdx.x & 31, row = row0 + lane;
        const float ca = a.coefficients[tile.step][0];
        const bool last = tile.step + 1 == a.steps, full = tile.step + 2 >= a.steps;
        float d_row = 0.0f;
        if (parts > 0 && (tile.what == 1 || (tile.what == 2 && !tile.tall))) d_row = __ldcg(a.w.diags + tile.diag + row);
#pragma unroll 1
        for (int part = 0; part < parts; ++part) {
            if (here(tile, part)) {
                const int c0 = col + 32 * part;
                column = next_column;
                if (tile.what > 0) {
                    if (!mbar_wait_warp(bar, phase, a.wait_ns)) return false;
                    phase ^= 1;
                }
                __syncwarp();
                uint32_t h[16];
                if (tile.what < 2) {
                    uint32_t low[16];
                    if (tile.what == 1) {
                        get_row(place, lane, h);
                        if constexpr (FINE) get_row(place + kPartBytes, lane, low);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float raw[16];
                        tmem_load16(src + 32 * part + 16 * k, raw);
                        // (a warp's 32 x 32 are on the diagonal as a whole, or off)
                        square16(tile, row, c0 == row0, d_row, raw, h + 8 * k, low + 8 * k, 16 * k);
                    }
                    // above the diagonal's blocks: the transposed part too
                    const bool mirror = c0 / kBlock > row0 / kBlock;
                    const int y = c0 / kPanel * tile.pitch + row0, y_across = row0 / kPanel * tile.pitch + c0;
                    put_row(place, lane, h);
                    if constexpr (FINE) put_row(place + kPartBytes, lane, low);
                    else if (mirror) put_across(place + kPartBytes, h);
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        store_part(map, c0 % kPanel, tile.out + y, place);
                        if constexpr (FINE) store_part(map, c0 % kPanel, tile.out_low + y, place + kPartBytes);
                        else if (mirror) store_part(map, row0 % kPanel, tile.out + y_across, place + kPartBytes);
                        stores_commit();
                    }
                    if (FINE && mirror) {               // (both places once more)
                        if (lane == 0) stores_read();
                        __syncwarp();
                        put_across(place, h);
                        put_across(place + kPartBytes, low);
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0) {
                            store_part(map, row0 % kPanel, tile.out + y_across, place);
                            store_part(map, row0 % kPanel, tile.out_low + y_across, place + kPartBytes);
                            stores_commit();
                        }
                    }
                } else if (!last) {
                    uint32_t low[16];
                    get_row(place, lane, h);
                    get_row(place + kPartBytes, lane, low);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float raw[16];
                        tmem_load16(src + 32 * part + 16 * k, raw);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const F2 v = next_x(tile, 16 * k + 2 * i, F2(raw[2 * i], raw[2 * i + 1]), h[8 * k + i], low[8 * k + i], d_row, ca, full);
                            h[8 * k + i] = pack_half(v);
                            low[8 * k + i] = pack_half(fma2(halves(h[8 * k + i]), F2(-1.0f), v) * F2(kLow));
                        }
                    }
                    put_row(place, lane, h);
                    put_row(place + kPartBytes, lane, low);
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        const int y = c0 / kPanel * tile.pitch + row0;
                        store_part(map, c0 % kPanel, tile.out + y, place);
                        store_part(map, c0 % kPanel, tile.out_low + y, place + kPartBytes);
                        stores_commit();
                    }
                } else {
                    uint32_t low[16];
                    get_row(place, lane, h);
                    get_row(place + kPartBytes, lane, low);
                    float v[32];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float raw[16];
                        tmem_load16(src + 32 * part + 16 * k, raw);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            (next_x(tile, 16 * k + 2 * i, F2(raw[2 * i], raw[2 * i + 1]), h[8 * k + i], low[8 * k + i], d_row, ca, full) * F2(1.0f / kScaleX))
                                .get(v[16 * k + 2 * i], v[16 * k + 2 * i + 1]);
                    }
                    __syncwarp();
                    const Item &it = a.w.items[tile.which];
                    if (a.theta) step_theta(it, a.decay, place, row0, c0, v);
                    else write_out(it, place, row0, c0, v);
                    // (the next load into this place comes behind what was read there)
                    fence_async_shared();
                }
                __syncwarp();
            }
            fetch(tile, part + 1);
        }
        return true;
    }
    // Two elements of the next X: a x + d x + (the product's sum), x by its two parts.
    __device__ __forceinline__ F2 next_x(const Tile &tile, int i, F2 sum, uint32_t hi, uint32_t low, float d_row, float ca, bool full) const
    {
        const F2 p = halves(hi), x = fma2(halves(low), F2(1.0f / kLow), p);
        F2 d(d_row);
        if (tile.tall) d = columns(i);
        return fma2(sum, F2(1.0f / kScaleB), fma2(d, FINE || full ? x : p, x * F2(ca)));
    }
};

template <bool FINE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
novak_orthogonalize_products_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ CUtensorMap map,
                                    const __grid_constant__ CUtensorMap part_map)
{
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (smem_addr(raw) + 1023) & ~1023u, places = stages + kStages * kStageBytes;
    Shared &sh = *reinterpret_cast<Shared *>(raw + (places - smem_addr(raw)) + kOutWarps * kPlaceBytes);
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
            mbar_init(smem_addr(&sh.ready[i]), 1);
            mbar_init(smem_addr(&sh.tile_empty[i]), 2 * kOutWarps + 3);      // who takes, who brings, and who issues
        }
        for (int i = 0; i < kOutWarps; ++i) mbar_init(smem_addr(&sh.part_full[i]), 1);
        mbar_init(smem_addr(&sh.want), 1);
        mbar_init(smem_addr(&sh.drained), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc_pair(smem_addr(&sh.tmem), 512);
    if (threadIdx.x == 32 * kLoadWarp) {
        prefetch_map(&map);
        prefetch_map(&part_map);
    }
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;
    start();

    bool ok = true;
    Ring<kRing> ring;
    // The next tile is in its place in the ring; to be given back when it is done with.
    const auto next = [&] {
        ok = mbar_wait_warp(smem_addr(&sh.tile_full[ring.slot]), ring.phase, a.wait_ns);
        if (!ok) {
            if (lane == 0) gave_up(a);
            return false;
        }
        return sh.tiles[ring.slot].what >= 0;
    };
    const auto release = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed(at_rank(smem_addr(&sh.tile_empty[ring.slot]), 0));
        ring.advance();
    };
    if (warp < kOutWarps) {
        const int group = warp / 4, quarter = warp % 4;
        Taking<FINE> taking{a, &part_map, places + warp * kPlaceBytes, smem_addr(&sh.part_full[warp]), 0, false, 0, 0, false, 0, 0, 0, 0.0f, 0.0f};
        for (uint32_t count = 0;; ++count) {
            const uint32_t buf = count & 1, ready = smem_addr(&sh.ready[ring.slot]);
            // (nobody waits longer than need be for what is stored)
            if (!__all_sync(0xffffffffu, mbar_try_now(smem_addr(&sh.tile_full[ring.slot]), ring.phase))) taking.tell();
            if (!next()) break;
            const Tile &tile = sh.tiles[ring.slot];
            const int quarter_columns = tile.columns / 4;
            taking.row0 = tile.row + static_cast<int>(rank) * kBlock + quarter * 32;
            taking.col = tile.col + group * quarter_columns;
            taking.parts = taking.row0 < tile.height ? quarter_columns / 32 : 0;
            // What the tile needs beside its products, on its way before they are awaited, and before the tile before has
            // arrived in memory, unless this one waits for that.
            if (!__all_sync(0xffffffffu, mbar_try_now(ready, ring.phase))) {
                taking.tell();
                ok = mbar_wait_warp(ready, ring.phase, a.wait_ns);
            }
            if (ok) {
                taking.fetch(tile, 0);
                taking.tell();
                ok = mbar_wait_warp(smem_addr(&sh.out_full[buf]), (count >> 1) & 1, a.wait_ns);
            }
            if (ok) {
                tcgen05_after_sync();
                ok = taking.take(tile, tmem + buf * 256 + group * quarter_columns + (static_cast<uint32_t>(quarter) * 32 << 16));
            }
            if (!ok) {
                if (lane == 0) gave_up(a);
                taking.untold = true;           // (parts may be on their way to memory)
                taking.told = 0;
                break;
            }
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(at_rank(smem_addr(&sh.out_empty[buf]), 0));
            taking.untold = true;
            taking.told_which = tile.which;
            taking.told = tile.announced;
            taking.own_stores = tile.what < 2 || tile.step + 1 == a.steps;
            release();
        }
        taking.tell();
    } else if (warp == kLoadWarp) {
        Ring<kStages> at;
        int64_t issued = 0;
        const uint32_t full0 = at_rank(smem_addr(&sh.full[0]), 0);
        for (;;) {
            const uint32_t ready = smem_addr(&sh.ready[ring.slot]);
            if (!ok || !next()) break;
            const Tile tile = sh.tiles[ring.slot];
            release();
            if (lane == 0) {
                ok = wait_parts(a, a.w.done + tile.which, tile.need);
                // (what other SMs have stored is there for tensor copies, this warp's and those of the warps that wait for `ready`)
                asm volatile("fence.proxy.async;" ::: "memory");
                if (ok) mbar_arrive(ready);
                const int boxes = tile.columns / 128, all = (FINE ? 3 : 1) * tile.steps;
                int ya = tile.a + static_cast<int>(rank) * tile.a_rank, yb = tile.b + static_cast<int>(rank) * tile.b_rank;
                for (int i = 0; ok && i < all; ++i, ya += tile.a_step, yb += tile.b_step) {
                    // fine: first parts, then the first by the second, then the second by the first
                    if (FINE && i == tile.steps) {
                        ya -= tile.steps * tile.a_step;
                        yb += tile.b_low - tile.steps * tile.b_step;
                    }
                    if (FINE && i == 2 * tile.steps) {
                        ya += tile.a_low - tile.steps * tile.a_step;
                        yb -= tile.b_low + tile.steps * tile.b_step;
                    }
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
                    if (rank == 0 && i == max(all - 12, 0)) mbar_arrive(smem_addr(&sh.want));
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
        while (ok && next()) {
            const Tile tile = sh.tiles[ring.slot];
            release();
            const uint32_t buf = count & 1, d = tmem + buf * 256;
            const bool a_across = tile.descriptor >> 15 & 1, b_across = tile.descriptor >> 16 & 1;
            const uint32_t a_next = a_across ? 2048 >> 4 : 32 >> 4, b_next = b_across ? 2048 >> 4 : 32 >> 4;
            const uint64_t a0 = operand_desc(stages, kBoxBytes, 1024), b0 = operand_desc(stages + 2 * kBoxBytes, kBoxBytes, 1024);
            ok = mbar_wait_warp(smem_addr(&sh.out_empty[buf]), ((count >> 1) & 1) ^ 1, a.wait_ns);
            tcgen05_after_sync();
            const int all = (FINE ? 3 : 1) * tile.steps;
            for (int i = 0; ok && i < all; ++i) {
                ok = mbar_wait_warp(smem_addr(&sh.full[at.slot]), at.phase, a.wait_ns);
                if (!ok) break;
                tcgen05_after_sync();
                const uint64_t a_at = a0 + at.slot * (kStageBytes >> 4), b_at = b0 + at.slot * (kStageBytes >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_pair_bf16(d, a_at + k * a_next, b_at + k * b_next, tile.descriptor, i > 0 || k > 0);
                    mma_commit_pair(smem_addr(&sh.empty[at.slot]));
                    if (i == all - 1) mma_commit_pair(smem_addr(&sh.out_full[buf]));
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
        bool more = true;
        // The next tile is taken some 6000 cycles before this one's last operands are on their way, which finding
        // out what it is takes, and not before: with fewer tiles than pairs everybody is to have one.
        for (uint32_t taken = 0; more && ok; ++taken) {
            int64_t t = 0;
            if (taken > 0 && !mbar_wait_warp(smem_addr(&sh.want), (taken - 1) & 1, a.wait_ns)) {
                ok = false;
                if (lane == 0) gave_up(a);
            }
            if (lane == 0) t = !ok || load_acquire(&a.control->failed) ? all : atomicAdd(&a.control->ticket, 1u);
            t = __shfl_sync(0xffffffffu, t, 0);
            more = t < all;
            Tile tile{};
            if (more) tile = tile_at<FINE>(a, t);
            else tile.what = -1;
            if (!mbar_wait_warp(smem_addr(&sh.tile_empty[ring.slot]), ring.phase ^ 1, a.wait_ns)) {
                ok = false;
                if (lane == 0) gave_up(a);
                break;
            }
            // (every lane has all of its words: lane i sends word i to both CTAs)
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < kTileWords; ++i)
                if (lane == i) word = tile_word(tile, i);
            for (uint32_t r = 0; r < 2; ++r) {
                const uint32_t bar = at_rank(smem_addr(&sh.tile_full[ring.slot]), r);
                if (lane == 0) mbar_expect_at(bar, sizeof(Tile));
                __syncwarp();
                if (lane < kTileWords) send_word(at_rank(smem_addr(&sh.tiles[ring.slot]), r) + 4 * lane, word, bar);
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

// Matrices that have a place in the workspace: not those that stay in shared memory (in a test of the waits, which those
// do without: all).
static bool placed(int64_t rows, int64_t cols, bool all) { return rows > 0 && cols > 0 && (all || small_ctas(rows, cols) == 0); }

// The matrices of a call in groups that use one workspace after another: f(first one, first one behind, bytes).  A group is as many
// as fit kGroupBytes, or one that does not: a step of all of a model's matrices takes no more memory than that.
// What a matrix comes to does not depend on its group.  (Groups' ends cost the last tiles of 15 products each, about 1 %: 24 of
// 4096 x 4096 in groups of six 31 ms.)  false: more than can be addressed.
constexpr size_t kGroupBytes = size_t(1) << 30;
template <typename F> bool for_groups(const int64_t *rows, const int64_t *cols, int n, bool fine, bool all, const F &f)
{
    Layout total, l;
    Item it{};
    int first = 0, count = 0;
    for (int i = 0; i < n; ++i) {
        if (!placed(rows[i], cols[i], all)) continue;
        if (!place(total, rows[i], cols[i], fine, it)) return false;
        Layout longer = l;
        place(longer, rows[i], cols[i], fine, it);
        finish_layout(longer, count + 1);
        if (count > 0 && longer.bytes > kGroupBytes) {
            f(first, i, l.bytes);
            longer = Layout();
            place(longer, rows[i], cols[i], fine, it);
            finish_layout(longer, 1);
            first = i;
            count = 0;
        }
        l = longer;
        ++count;
    }
    if (count > 0) f(first, n, l.bytes);
    return true;
}

size_t orthogonalize_bytes(const int64_t *rows, const int64_t *cols, int n, bool fine, bool all)
{
    size_t most = 0;
    if (!for_groups(rows, cols, n, fine, all, [&](int, int, size_t bytes) { most = std::max(most, bytes); })) return 0;
    for (int i = 0; i < n && most == 0; ++i)
        if (rows[i] > 0 && cols[i] > 0) most = kLeastBytes;
    return most;
}

cudaError_t orthogonalize_gave_up(unsigned *count, cudaStream_t stream)
{
    cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_orthogonalize_gave_up, sizeof *count, 0, cudaMemcpyDeviceToHost, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

// Matrices [begin, end) of a call by the tensor cores; `withheld`: of the group's tiles, whose number becomes `tiles_of_it`.
static cudaError_t launch_group(const OrthArgs &a, int begin, int end, int64_t withheld, int64_t &tiles_of_it, cudaStream_t stream);

cudaError_t launch_orthogonalize(const OrthArgs &a, cudaStream_t stream)
{
    const Momentum mo{a.m != nullptr, a.nesterov, a.momentum};
    const bool f32 = a.type == NOVAK_TYPE_F32, all = a.withheld >= 0;
    SmallArgs small{};
    for (int k = 0; k < a.steps; ++k)
        for (int i = 0; i < 3; ++i) small.coefficients[k][i] = a.coefficients[k][i];
    small.steps = a.steps;
    small.theta = a.out == nullptr;
    small.decay = a.decay;
    small.eps = static_cast<float>(a.eps);
    small.mo = mo;
    cudaError_t e = cudaSuccess;
    if (!all) e = f32 ? launch_small<0, 1>(a, small, stream) : launch_small<1, 1>(a, small, stream);
    if (!all && e == cudaSuccess) e = f32 ? launch_small<0, kSmallCluster>(a, small, stream) : launch_small<1, kSmallCluster>(a, small, stream);
    int64_t withheld = a.withheld;
    for_groups(a.rows, a.cols, a.n, a.fine, all, [&](int begin, int end, size_t) {
        int64_t tiles = 0;
        if (e == cudaSuccess) e = launch_group(a, begin, end, withheld, tiles, stream);
        withheld = withheld >= tiles ? withheld - tiles : -1;
    });
    return e;
}

static cudaError_t launch_group(const OrthArgs &a, int begin, int end, int64_t withheld, int64_t &tiles_of_it, cudaStream_t stream)
{
    const Momentum mo{a.m != nullptr, a.nesterov, a.momentum};
    const bool f32 = a.type == NOVAK_TYPE_F32, all = a.withheld >= 0;
    const auto here = [&](int i) { return placed(a.rows[i], a.cols[i], all); };
    cudaError_t e = cudaSuccess;
    Layout l;
    Item it{};
    int n = 0, first_of[3] = {};
    int64_t tiles[3][2] = {};           // of a step, by product: of 256 columns, and of 128
    for (int i = begin; i < end; ++i)
        if (here(i)) {
            place(l, a.rows[i], a.cols[i], a.fine, it);
            for (int what = 0; what < 3; ++what)
                for (int narrow = 0; narrow < 2; ++narrow) tiles[what][narrow] += tiles_of(it, what, narrow ? 128 : 256);
            ++n;
        }
    finish_layout(l, n);
    uint8_t *base = static_cast<uint8_t *>(a.work);
    const Work w{reinterpret_cast<__half *>(base), reinterpret_cast<float *>(base + l.diags), reinterpret_cast<Item *>(base + l.items),
                 reinterpret_cast<double *>(base + l.partial), reinterpret_cast<unsigned *>(base + l.done)};
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
    tiles_of_it = static_cast<int64_t>(p.first[3]) * a.steps;
    Layout again;
    HostItems<kMostItems> items{};
    int first = 0, count = 0;
    const auto send = [&] {
        const dim3 chunks(static_cast<unsigned>(again.chunks - items.item[0].chunk));
        const auto with = [&](auto few, auto kernel) {
            std::copy_n(items.item, count, few.item);
            return launch(kernel, chunks, kThreads, 0, stream, few, first, count, w, p.control, mo);
        };
        const cudaError_t e = count <= 8    ? with(HostItems<8>{}, f32 ? novak_orthogonalize_norm_kernel<0, 8> : novak_orthogonalize_norm_kernel<1, 8>)
                              : count <= 40 ? with(HostItems<40>{}, f32 ? novak_orthogonalize_norm_kernel<0, 40> : novak_orthogonalize_norm_kernel<1, 40>)
                                            : with(HostItems<kMostItems>{}, f32 ? novak_orthogonalize_norm_kernel<0, kMostItems> : novak_orthogonalize_norm_kernel<1, kMostItems>);
        first += count;
        count = 0;
        return e;
    };
    for (int i = begin; i < end && e == cudaSuccess; ++i) {
        if (!here(i)) continue;
        place(again, a.rows[i], a.cols[i], a.fine, it);
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
        if (count == kMostItems) e = send();
    }
    if (e == cudaSuccess && count > 0) e = send();
    if (e == cudaSuccess)
        e = launch(f32 ? novak_orthogonalize_start_kernel<0> : novak_orthogonalize_start_kernel<1>, 
                   dim3(static_cast<unsigned>(std::min<int64_t>(l.units, 148 * 4))), kThreads, 0, stream, w, n, l.units, mo, static_cast<float>(a.eps), a.fine ? 1.0f : kScaleLow);
    if (e != cudaSuccess) return e;

    for (int k = 0; k < a.steps; ++k)
        for (int i = 0; i < 3; ++i) p.coefficients[k][i] = a.coefficients[k][i];
    p.decay = a.decay;
    p.theta = a.out == nullptr;
    p.withheld = withheld;
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
    CUtensorMap part_map;
    const cuuint32_t part_box[2] = {32, 32};
    if (encode(&part_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, part_box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> asked[2] = {};
    const auto kernel = a.fine ? novak_orthogonalize_products_kernel<true> : novak_orthogonalize_products_kernel<false>;
    e = ask_shared_memory(kernel, kSmemBytes, asked[a.fine]);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3(static_cast<unsigned>(2 * std::min<int64_t>(kPairs, most))), kTcThreads, kSmemBytes,
                  stream, p, map, part_map);
}

}  // namespace novak
