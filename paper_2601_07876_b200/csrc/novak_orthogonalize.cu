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
    float step;
    int unused;
};
static_assert(sizeof(Item) == 104, "as the host fills it");

struct Work {
    __half *panels;
    float *diags;
    Item *items;
    double *partial;            // per unit
    float2 *scale;              // per matrix: G is multiplied by one, then by the other
    unsigned *arrived;          // per matrix
};

struct Layout {
    int64_t panel_rows = 0, diag_floats = 0, units = 0;
    size_t diags, items, partial, scale, arrived, bytes;
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
    if (l.panel_rows + 3 * x + 2 * s > INT_MAX) return false;
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
    l.bytes = l.arrived + round_up(n * sizeof(unsigned));
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
    static constexpr int kMost = 256;
    Item item[kMost];
};

__global__ void novak_orthogonalize_items_kernel(const __grid_constant__ HostItems from, int first, int count, Work w)
{
    start();
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        w.items[first + i] = from.item[i];
        w.arrived[first + i] = 0;
    }
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

// ---- the products, simply ----------------------------------------------------------
struct Phase {
    int what;                   // 0: A = X X^T; 1: B = b A + c A^2; 2: X <- a X + B X
    int turn;                   // which of X's two places is read
    float a, b, c;
    int full;                   // diag(B) multiplies both parts of X
    int last;                   // X goes out
    float decay;
    int theta;
};

__device__ __forceinline__ float panel_at(const __half *p, int base, int pitch, int row, int col)
{
    return __half2float(p[(static_cast<int64_t>(base) + static_cast<int64_t>(col / kPanel) * pitch + row) * kPanel + col % kPanel]);
}

__global__ void __launch_bounds__(kThreads) novak_orthogonalize_plain_kernel(Work w, int n, Phase ph)
{
    __shared__ float sa[16][65], sb[16][65];
    start();
    for (int which = 0; which < n; ++which) {
        const Item &it = w.items[which];
        const int height = ph.what == 2 ? it.x_pitch : it.s_pitch;
        const int width = pad_to(ph.what == 2 ? it.cols : it.side, kPanel);
        const int depth = ph.what == 0 ? (it.tall ? it.rows : it.cols) : it.side;
        const int tiles_x = width / 64, tiles = tiles_x * (height / 64);
        for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            const int r0 = tile / tiles_x * 64, c0 = tile % tiles_x * 64, ty = threadIdx.x / 16, tx = threadIdx.x % 16;
            float acc[4][4] = {};
            for (int k0 = 0; k0 < depth; k0 += 16) {
                __syncthreads();
                for (int e = threadIdx.x; e < 1024; e += kThreads) {
                    const int i = e % 64, k = e / 64, kk = k0 + k;
                    const int x = it.x[ph.turn];
                    float a, b;
                    if (ph.what == 0) {
                        const bool ia = r0 + i < it.side, ib = c0 + i < it.side;
                        a = !ia ? 0.0f : it.tall ? panel_at(w.panels, x, it.x_pitch, kk, r0 + i) : panel_at(w.panels, x, it.x_pitch, r0 + i, kk);
                        b = !ib ? 0.0f : it.tall ? panel_at(w.panels, x, it.x_pitch, kk, c0 + i) : panel_at(w.panels, x, it.x_pitch, c0 + i, kk);
                    } else if (ph.what == 1) {
                        a = panel_at(w.panels, it.gram, it.s_pitch, r0 + i, kk);
                        b = panel_at(w.panels, it.gram, it.s_pitch, kk, c0 + i);
                    } else if (!it.tall) {
                        a = panel_at(w.panels, it.poly, it.s_pitch, r0 + i, kk);
                        b = panel_at(w.panels, x, it.x_pitch, kk, c0 + i);
                    } else {
                        a = panel_at(w.panels, x, it.x_pitch, r0 + i, kk);
                        b = panel_at(w.panels, it.poly, it.s_pitch, kk, c0 + i);
                    }
                    sa[k][i] = kk < depth ? a : 0.0f;
                    sb[k][i] = kk < depth ? b : 0.0f;
                }
                __syncthreads();
                for (int k = 0; k < 16; ++k)
                    for (int i = 0; i < 4; ++i)
                        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
            }
            float *da = w.diags + it.diag, *db = da + it.s_pitch;
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) {
                    const int r = r0 + ty * 4 + i, c = c0 + tx * 4 + j;
                    const int64_t s_at = (static_cast<int64_t>(c / kPanel) * it.s_pitch + r) * kPanel + c % kPanel;
                    if (ph.what == 0) {
                        float v = acc[i][j] * (1.0f / (kScaleX * kScaleX));
                        if (r == c) {
                            da[r] = v;
                            v = 0.0f;
                        }
                        w.panels[static_cast<int64_t>(it.gram) * kPanel + s_at] = __float2half_rn(v * kScaleA);
                    } else if (ph.what == 1) {
                        const float off = __half2float(w.panels[static_cast<int64_t>(it.gram) * kPanel + s_at]) * (1.0f / kScaleA);
                        const float sq = acc[i][j] * (1.0f / (kScaleA * kScaleA));
                        float v = ph.b * off + ph.c * (sq + (da[r] + da[c]) * off);
                        if (r == c) {
                            db[r] = ph.b * da[r] + ph.c * (sq + da[r] * da[r]);
                            v = 0.0f;
                        }
                        w.panels[static_cast<int64_t>(it.poly) * kPanel + s_at] = __float2half_rn(v * kScaleB);
                    } else {
                        const int64_t at = (static_cast<int64_t>(c / kPanel) * it.x_pitch + r) * kPanel + c % kPanel;
                        const float hi = __half2float(w.panels[static_cast<int64_t>(it.x[ph.turn]) * kPanel + at]);
                        const float lo = __half2float(w.panels[static_cast<int64_t>(it.low) * kPanel + at]) * (1.0f / kScaleLow);
                        const float d = db[it.tall ? c : r], x = hi + lo;
                        float v = fmaf(acc[i][j], 1.0f / kScaleB, fmaf(d, ph.full ? x : hi, ph.a * x));
                        if (ph.last) {
                            v *= 1.0f / kScaleX;
                            if (r < it.rows && c < it.cols) {
                                if (ph.theta) {
                                    float *t = static_cast<float *>(it.out) + static_cast<int64_t>(r) * it.cols + c;
                                    *t = fmaf(-it.step, v, ph.decay * *t);
                                } else {
                                    store_param(it.out, NOVAK_TYPE_BF16, r * it.out_stride + c, v);
                                }
                            }
                        } else {
                            split(v, w.panels[static_cast<int64_t>(it.x[1 - ph.turn]) * kPanel + at],
                                  w.panels[static_cast<int64_t>(it.low) * kPanel + at]);
                        }
                    }
                }
        }
    }
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

cudaError_t orthogonalize_gave_up(unsigned *count, cudaStream_t)
{
    *count = 0;
    return cudaSuccess;
}

cudaError_t launch_orthogonalize(const OrthArgs &a, cudaStream_t stream)
{
    Layout l;
    Item it{};
    int n = 0;
    for (int i = 0; i < a.n; ++i)
        if (a.rows[i] > 0 && a.cols[i] > 0) {
            place(l, a.rows[i], a.cols[i], it);
            ++n;
        }
    if (n == 0) return cudaSuccess;
    finish_layout(l, n);
    uint8_t *base = static_cast<uint8_t *>(a.work);
    const Work w{reinterpret_cast<__half *>(base), reinterpret_cast<float *>(base + l.diags), reinterpret_cast<Item *>(base + l.items),
                 reinterpret_cast<double *>(base + l.partial), reinterpret_cast<float2 *>(base + l.scale),
                 reinterpret_cast<unsigned *>(base + l.arrived)};
    Layout again;
    HostItems items;
    int first = 0, count = 0;
    const auto send = [&] {
        const cudaError_t e = launch(novak_orthogonalize_items_kernel, dim3(1), kThreads, 0, stream, items, first, count, w);
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
    for (int k = 0; k < a.steps; ++k)
        for (int what = 0; what < 3 && e == cudaSuccess; ++what) {
            const Phase ph{what, k & 1, a.coefficients[k][0], a.coefficients[k][1], a.coefficients[k][2], k + 2 >= a.steps,
                           k + 1 == a.steps, a.decay, a.out == nullptr};
            e = launch(novak_orthogonalize_plain_kernel, dim3(148 * 4), kThreads, 0, stream, w, n, ph);
        }
    return e;
}

}  // namespace novak
