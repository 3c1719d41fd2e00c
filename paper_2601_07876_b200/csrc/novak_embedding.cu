// Token embedding, out[t] = scale table[ids[t]], and its gradient, the sum of dout's rows
// over the tokens of an id.
//
// Looking up is reading and writing rows; what bounds it is HBM, and for few tokens latency, so
// that long rows are cut among warps.
//
// The gradient of a whole table is mostly zeros to be written; the rest is to bring each id's
// tokens together in an order that goes by their places alone.  No sort of all ids by digits:
// ids are dealt out by their low bits to some hundred CTAs (words of like frequency have like
// numbers; so they go to different ones), and each CTA looks through all ids, which L2
// holds, for its own.  It counts its rows' tokens and those of the CTAs before it, which says where
// its tokens lie in the order of all, and
//   writes zeros for rows without tokens (or leaves them, where the sum is added),
//   sums rows of up to 64 tokens by itself, a warp 256 columns,
//   leaves the tokens of longer ones, in order, to the second kernel, which cuts the order of
//   all tokens into pieces of 64 and gives each a CTA; the last one of a row's pieces to be done
//   adds their sums up in order.
// So it is one pass over dout and one over the table, however unevenly words occur.
#include <algorithm>
#include <climits>

#include "novak_ops.cuh"

namespace novak {
namespace {

__device__ __forceinline__ int64_t id_at(const void *ids, int type, int64_t t)
{
    return type == NOVAK_ID_I32 ? static_cast<const int32_t *>(ids)[t] : static_cast<const int64_t *>(ids)[t];
}

// ---- looking up ----------------------------------------------------------------------
constexpr int kLookThreads = 256, kLookGroups = 4;      // groups of 8 elements on their way per lane

struct LookArgs : EmbedArgs {
    int lanes, parts;       // lanes of a row, a power of two; pieces of lanes * 8 * kLookGroups elements that it is cut into
};

template <int TABLE, int OUT, bool ALIGNED>
__global__ void __launch_bounds__(kLookThreads) novak_embedding_kernel(LookArgs a)
{
    using T = typename Elem<TABLE>::T;
    using O = typename Elem<OUT>::T;
    const int lane = threadIdx.x % a.lanes;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kLookThreads + threadIdx.x) / a.lanes;
    const int64_t t = unit <= INT_MAX ? static_cast<unsigned>(unit) / static_cast<unsigned>(a.parts) : unit / a.parts, part = unit - t * a.parts;
    const void *begin = a.table.ptr, *end = end_of(static_cast<const T *>(a.table.ptr), a.table.stride, a.vocab, a.cols);
    start();
    if (t >= a.tokens) return;          // (a warp has one row's lanes where it matters that all are here)
    const int64_t id = id_at(a.ids, a.id_type, t);
    const bool there = id >= 0 && id < a.vocab;
    const int64_t col = part * a.lanes * 8 * kLookGroups + lane * 8;
    const T *row = static_cast<const T *>(a.table.ptr) + (there ? id : 0) * a.table.stride + col;
    O *out = static_cast<O *>(a.out.ptr) + t * a.out.stride + col;
    Fetch<TABLE, ALIGNED> raw[kLookGroups];
    int n[kLookGroups];
#pragma unroll
    for (int i = 0; i < kLookGroups; ++i) {
        n[i] = static_cast<int>(max(min(a.cols - col - static_cast<int64_t>(i) * a.lanes * 8, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
        raw[i].zero();
        if (there) raw[i].load(row + i * a.lanes * 8, n[i], begin, end);
    }
    const F2 scale(a.scale);
#pragma unroll
    for (int i = 0; i < kLookGroups; ++i) {
        F2 v[4];
        raw[i].eight().get(v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = there ? v[k] * scale : F2(0.0f);
        Eight<OUT> e;
        e.set(v);
        store_eight<ALIGNED>(out + i * a.lanes * 8, e, n[i]);
    }
}

// ---- the gradient --------------------------------------------------------------------
constexpr int kOwnThreads = 512, kOwnRows = 4096;       // rows of the table per CTA at most
constexpr int kList = 2048, kBitWords = 2048;           // tokens that a CTA keeps in shared memory; words of its bit map
constexpr int kPiece = 64;                              // tokens in a piece of the second kernel
constexpr int kSlice = 1024, kSumThreads = 256;         // columns of a CTA there
constexpr int kFewTokens = 256;                         // up to which there is no second kernel

struct Segment {            // of a token in the order of all, if it is its row's second kernel's
    int row, start, count, token;
};

struct GradArgs : EmbedGradArgs {
    int shift;              // CTA p has the ids whose low `shift` bits are p
    int longest;            // tokens of a row that are summed at once
    int lanes;              // of a row (ALIGNED), of 8 columns each
    int slices;             // of the columns, in the second kernel
    int group;              // its threads per token
    int *list;              // tokens, for CTAs that have more than kList
    Segment *order;
    int *counts;            // [piece][slice]: sums that are done, where a row begins in that piece
    int *valid;             // tokens in all
    float *partial;         // [piece][2][cols]: of a row that began before, of one that begins here
};

// Sums over the CTA in the order of threads: those before this one, and all.
__device__ __forceinline__ int scan(int x, int *scratch, int &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = s;
    __syncthreads();
    int before = 0;
    all = 0;
    for (int w = 0; w < kOwnThreads / 32; ++w) {
        const int y = scratch[w];
        if (w < warp) before += y;
        all += y;
    }
    return before + s - x;
}

// Adds the lanes that are `mine` to counters[row], lanes of one row together (an id may be on
// every lane); the place of each among what the counter had and the lanes before it.
__device__ __forceinline__ int count_rows(bool mine, int row, int *counters)
{
    unsigned left = __ballot_sync(0xffffffffu, mine);
    const int lane = threadIdx.x & 31;
    int place = 0;
    while (left) {
        const int leader = __ffs(static_cast<int>(left)) - 1, of = __shfl_sync(0xffffffffu, row, leader);
        const unsigned same = __ballot_sync(0xffffffffu, mine && row == of);
        int base = 0;
        if (lane == leader) base = atomicAdd(counters + of, __popc(same));
        base = __shfl_sync(0xffffffffu, base, leader);
        if (mine && row == of) place = base + __popc(same & ((1u << lane) - 1));
        left &= ~same;
    }
    return place;
}

// Eight columns of the sum over `count` tokens.
template <int TYPE, bool ALIGNED>
__device__ __forceinline__ void sum_tokens(const EmbedGradArgs &a, const int *tokens, int count, int64_t col, int n, const void *begin,
                                           const void *end, F2 (&sum)[4])
{
    using T = typename Elem<TYPE>::T;
    constexpr int kAhead = !ALIGNED ? 2 : TYPE == NOVAK_TYPE_F32 ? 4 : 8;
    const T *base = static_cast<const T *>(a.dout.ptr) + col;
    for (int j = 0; j < count; j += kAhead) {
        Fetch<TYPE, ALIGNED> raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            raw[k].zero();
            if (j + k < count) raw[k].load(base + tokens[j + k] * a.dout.stride, n, begin, end);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            F2 v[4];
            raw[k].eight().get(v);
            if (j + k < count)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = sum[i] + v[i];
        }
    }
}

// The table's eight elements at p from their sum.
template <int GRAD, bool ALIGNED>
__device__ __forceinline__ void put_sum(const EmbedGradArgs &a, typename Elem<GRAD>::T *p, int n, const F2 (&sum)[4], const void *begin, const void *end)
{
    const F2 scale(a.scale);
    F2 v[4];
    if (a.add) {
        Fetch<GRAD, ALIGNED> old;
        old.zero();
        old.load(p, n, begin, end);
        old.eight().get(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fma2(sum[i], scale, v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = sum[i] * scale;
    }
    Eight<GRAD> e;
    e.set(v);
    store_eight<ALIGNED>(p, e, n);
}

struct OwnShared {
    int counts[kOwnRows], starts[kOwnRows];
    int2 found[kList];          // row, token
    int list[kList];
    uint32_t bits[kBitWords];
    int scratch[kOwnThreads / 32];
    int n;
};

template <int TYPE, int GRAD, bool ALIGNED>
__global__ void __launch_bounds__(kOwnThreads, 2) novak_embedding_grad_kernel(GradArgs a)
{
    using G = typename Elem<GRAD>::T;
    extern __shared__ uint8_t raw_shared[];
    OwnShared &sh = *reinterpret_cast<OwnShared *>(raw_shared);
    const int64_t own = blockIdx.x, low = (int64_t(1) << a.shift) - 1;
    const int rows = static_cast<int>((a.vocab - own + low) >> a.shift);        // ids own, own + 2^shift, ...
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < rows; i += kOwnThreads) sh.counts[i] = 0;
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    start();

    // ---- all ids: how many are this CTA's, by row, and how many belong to CTAs before it
    int before = 0, valid = 0;
    const auto look = [&](auto &&take) {
        constexpr int kAhead = 8;
        for (int64_t t0 = 0; t0 < a.tokens; t0 += kAhead * kOwnThreads) {
            int64_t id[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t t = t0 + k * kOwnThreads + threadIdx.x;
                id[k] = t < a.tokens ? id_at(a.ids, a.id_type, t) : -1;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) take(id[k], static_cast<int>(t0 + k * kOwnThreads + threadIdx.x));
        }
    };
    look([&](int64_t id, int t) {
        const bool there = id >= 0 && id < a.vocab;
        valid += there;
        before += there && (id & low) < own;
        const bool mine = there && (id & low) == own;
        const unsigned m = __ballot_sync(0xffffffffu, mine);
        if (m == 0) return;
        const int row = static_cast<int>(id >> a.shift);
        count_rows(mine, row, sh.counts);
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, __popc(m));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(m & ((1u << lane) - 1));
        if (mine && at < kList) sh.found[at] = make_int2(row, t);
    });
    int all;
    scan(before, sh.scratch, all);
    before = all;
    if (own == 0) {
        scan(valid, sh.scratch, all);
        if (threadIdx.x == 0) *a.valid = all;
    }
    __syncthreads();
    const int n = sh.n;
    int *list = n <= kList ? sh.list : a.list + before;

    // ---- where each row's tokens begin
    {
        constexpr int kEach = kOwnRows / kOwnThreads;
        const int first = threadIdx.x * kEach;
        int sum = 0;
        if (first < rows)
            for (int i = first; i < min(first + kEach, rows); ++i) sum += sh.counts[i];
        int at = scan(sum, sh.scratch, all);
        if (first < rows)
            for (int i = first; i < min(first + kEach, rows); ++i) {
                sh.starts[i] = at;
                at += sh.counts[i];
            }
    }
    __syncthreads();

    // ---- the tokens, row by row: put there in any order (counts go down to 0, starts up to the ends) ...
    const auto put = [&](bool mine, int row, int t) {
        if (__any_sync(0xffffffffu, mine)) {
            const int place = count_rows(mine, row, sh.starts);
            if (mine) list[place] = t;
        }
    };
    if (n <= kList) {
        for (int i = warp * 32; i < n; i += kOwnThreads) {
            const int2 f = i + lane < n ? sh.found[i + lane] : make_int2(0, 0);
            put(i + lane < n, f.x, f.y);
        }
    } else {
        look([&](int64_t id, int t) { put(id >= 0 && id < a.vocab && (id & low) == own, static_cast<int>(id >> a.shift), t); });
    }
    __syncthreads();

    // ---- ... and then in order.  A warp has short rows, a lane up to two tokens: its place is the
    // number of tokens before it.
    for (int row = warp; row < rows; row += kOwnThreads / 32) {
        const int count = sh.counts[row];
        if (count < 2 || count > 64) continue;
        int *mine = list + sh.starts[row] - count;
        const int x = lane < count ? mine[lane] : INT_MAX, y = lane + 32 < count ? mine[lane + 32] : INT_MAX;
        int px = 0, py = 0;
        for (int j = 0; j < min(count, 32); ++j) {
            const int u = __shfl_sync(0xffffffffu, x, j), v = __shfl_sync(0xffffffffu, y, j);
            px += (u < x) + (v < x);
            py += (u < y) + (v < y);
        }
        __syncwarp();
        if (lane < count) mine[px] = x;
        if (lane + 32 < count) mine[py] = y;
    }
    // Long ones: the tokens as bits of a map, 65536 of them at a time.
    for (int row = 0; row < rows; ++row) {
        const int count = sh.counts[row];
        if (count <= 64) continue;                  // (the same for all threads)
        const int first = sh.starts[row] - count;
        const bool later = count > a.longest;       // the second kernel's
        int done = 0;
        for (int64_t t0 = 0; t0 < a.tokens && done < count; t0 += 32 * kBitWords) {
            __syncthreads();
            for (int i = threadIdx.x; i < kBitWords; i += kOwnThreads) sh.bits[i] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < count; i += kOwnThreads) {
                const int64_t t = list[first + i] - t0;
                if (t >= 0 && t < 32 * kBitWords) atomicOr(&sh.bits[t >> 5], 1u << (t & 31));
            }
            __syncthreads();
            constexpr int kEach = kBitWords / kOwnThreads;
            int bits = 0;
            for (int i = 0; i < kEach; ++i) bits += __popc(sh.bits[threadIdx.x * kEach + i]);
            int at = done + scan(bits, sh.scratch, all);
            done += all;
            for (int i = 0; i < kEach; ++i)
                for (uint32_t m = sh.bits[threadIdx.x * kEach + i]; m; m &= m - 1, ++at) {
                    const int t = static_cast<int>(t0) + (threadIdx.x * kEach + i) * 32 + __ffs(static_cast<int>(m)) - 1;
                    if (later) a.order[before + first + at] = Segment{static_cast<int>(own + (static_cast<int64_t>(row) << a.shift)), before + first, count, t};
                    else list[first + at] = t;      // (one map holds all tokens: nothing of the list is needed any more)
                }
        }
        if (later)
            for (int i = threadIdx.x; i < a.slices; i += kOwnThreads) a.counts[static_cast<int64_t>((before + first) / kPiece) * a.slices + i] = 0;
    }
    __syncthreads();

    // ---- the table's rows: groups of lanes, a piece of a row's columns each
    if (a.longest < INT_MAX)                // what the second kernel passes over
        for (int row = warp; row < rows; row += kOwnThreads / 32) {
            const int count = sh.counts[row];
            if (count <= a.longest)
                for (int i = lane; i < count; i += 32) a.order[before + sh.starts[row] - count + i].row = -1;
        }
    const int lanes = ALIGNED ? a.lanes : 32, groups = kOwnThreads / lanes, mine = threadIdx.x / lanes;
    const int64_t steps = (a.cols + 8 * lanes - 1) / (8 * lanes), units = steps * rows;
    using T = typename Elem<TYPE>::T;
    const void *begin = a.dout.ptr, *end = end_of(static_cast<const T *>(a.dout.ptr), a.dout.stride, a.tokens, a.cols);
    const void *out_begin = a.dtable.ptr, *out_end = end_of(static_cast<const G *>(a.dtable.ptr), a.dtable.stride, a.vocab, a.cols);
    for (int64_t u = mine; u < units; u += groups) {
        const int row = units <= INT_MAX ? static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(steps)) : static_cast<int>(u / steps);
        const int count = sh.counts[row];
        if (count > a.longest || (a.add && count == 0)) continue;
        const int64_t col = (u - row * steps) * 8 * lanes + threadIdx.x % lanes * 8;
        const int here = static_cast<int>(max(min(a.cols - col, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
        F2 sum[4] = {F2(0.0f), F2(0.0f), F2(0.0f), F2(0.0f)};
        if (!ALIGNED || here > 0) {
            sum_tokens<TYPE, ALIGNED>(a, list + sh.starts[row] - count, count, col, here, begin, end, sum);
            put_sum<GRAD, ALIGNED>(a, static_cast<G *>(a.dtable.ptr) + (own + (static_cast<int64_t>(row) << a.shift)) * a.dtable.stride + col, here,
                                   sum, out_begin, out_end);
        }
    }
}

// A piece of the order of all tokens, 1024 columns: of at most two rows, since each row here has more tokens than a
// piece has: one that began before, and one that begins here.
template <int TYPE, int GRAD, bool ALIGNED>
__global__ void __launch_bounds__(kSumThreads) novak_embedding_pieces_kernel(GradArgs a)
{
    using G = typename Elem<GRAD>::T;
    using T = typename Elem<TYPE>::T;
    __shared__ int tokens[kPiece];
    __shared__ __align__(16) float part[kSumThreads * 8];
    __shared__ Segment first;
    __shared__ int begins;
    __shared__ bool last;
    start();
    const int piece = blockIdx.x, slice = blockIdx.y, from = piece * kPiece;
    const int here = min(*a.valid - from, kPiece);
    if (here <= 0) return;
    if (threadIdx.x == 0) begins = kPiece;
    Segment s{-1, 0, 0, 0};
    __syncthreads();
    if (threadIdx.x < kPiece) {
        if (static_cast<int>(threadIdx.x) < here) s = a.order[from + threadIdx.x];
        tokens[threadIdx.x] = s.token;
        if (threadIdx.x == 0) first = s;
        if (s.row >= 0 && s.start == from + static_cast<int>(threadIdx.x)) begins = threadIdx.x;
    }
    __syncthreads();
    __shared__ Segment second;
    if (static_cast<int>(threadIdx.x) == begins) second = s;
    __syncthreads();
    const int group = a.group, subs = kSumThreads / group, sub = threadIdx.x / group, t = threadIdx.x % group;
    const int64_t col = static_cast<int64_t>(slice) * kSlice + t * 8;
    const int n = static_cast<int>(max(min(a.cols - col, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
    const void *begin = a.dout.ptr, *end = end_of(static_cast<const T *>(a.dout.ptr), a.dout.stride, a.tokens, a.cols);
    for (int kind = 0; kind < 2; ++kind) {
        const int at = kind ? begins : 0;
        if (kind ? begins == kPiece : first.row < 0 || begins == 0) continue;
        const Segment seg = kind ? second : first;
        const int count = min(seg.start + seg.count - from, kPiece) - at;
        // this piece: every group of threads its share of the tokens, then the groups in order
        F2 sum[4] = {F2(0.0f), F2(0.0f), F2(0.0f), F2(0.0f)};
        const int share = (count + subs - 1) / subs, begin_at = min(sub * share, count);
        sum_tokens<TYPE, ALIGNED>(a, tokens + at + begin_at, min(share, count - begin_at), col, n, begin, end, sum);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2 *>(part + threadIdx.x * 8 + 2 * i) = make_float2(sum[i].lo(), sum[i].hi());
        __syncthreads();
        const int64_t pitch = a.cols;
        for (int c = threadIdx.x; c < group * 8; c += kSumThreads) {
            float x = 0.0f;
            for (int i = 0; i < subs; ++i) x += part[i * group * 8 + c];
            const int64_t out = static_cast<int64_t>(slice) * kSlice + c;
            if (out < a.cols) a.partial[(2 * static_cast<int64_t>(piece) + kind) * pitch + out] = x;
        }
        // the last of the row's pieces to be done adds all of them up
        const int head = seg.start / kPiece, pieces = (seg.start + seg.count - 1) / kPiece - head + 1;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(a.counts + static_cast<int64_t>(head) * a.slices + slice, 1) + 1 == pieces;
        __syncthreads();
        if (!last) continue;
        __threadfence();
        for (int c = threadIdx.x; c < group * 8; c += kSumThreads) {
            const int64_t out = static_cast<int64_t>(slice) * kSlice + c;
            if (out >= a.cols) continue;
            const float *p = a.partial + (2 * static_cast<int64_t>(head) + 1) * pitch + out;
            float x = __ldcg(p);
#pragma unroll 16
            for (int i = 1; i < pieces; ++i) x += __ldcg(p + (2 * static_cast<int64_t>(i) - 1) * pitch);     // (of a row that began before)
            part[c] = x;
        }
        __syncthreads();
        if (threadIdx.x < group) {
            F2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = F2(part[threadIdx.x * 8 + 2 * i], part[threadIdx.x * 8 + 2 * i + 1]);
            G *p = static_cast<G *>(a.dtable.ptr) + static_cast<int64_t>(seg.row) * a.dtable.stride + col;
            put_sum<GRAD, ALIGNED>(a, p, n, v, a.dtable.ptr, end_of(static_cast<const G *>(a.dtable.ptr), a.dtable.stride, a.vocab, a.cols));
        }
        __syncthreads();
    }
}

// ---- host ---------------------------------------------------------------------------
constexpr size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

// The least power of two that is not below n, at most `most`.
int power(int64_t n, int most)
{
    int p = 1;
    while (p < n && p < most) p *= 2;
    return p;
}

struct GradLayout {
    int64_t pieces;
    int slices;
    size_t list, order, counts, valid, partial, bytes;
};

GradLayout layout_of(int64_t tokens, int64_t cols)
{
    GradLayout l{};
    const bool second = tokens > kFewTokens;
    l.pieces = second ? (tokens + kPiece - 1) / kPiece : 0;
    l.slices = static_cast<int>((cols + kSlice - 1) / kSlice);
    l.list = 0;
    l.order = l.list + round_up((tokens > kList ? tokens : 0) * sizeof(int));
    l.counts = l.order + round_up((second ? tokens : 0) * sizeof(Segment));
    l.valid = l.counts + round_up(l.pieces * l.slices * sizeof(int));
    l.partial = l.valid + round_up(sizeof(int));
    l.bytes = l.partial + round_up(2 * l.pieces * cols * sizeof(float));
    return l;
}

template <int TYPE, int GRAD, bool ALIGNED> cudaError_t launch_grad(const GradArgs &g, int64_t pieces, cudaStream_t stream)
{
    const auto kernel = novak_embedding_grad_kernel<TYPE, GRAD, ALIGNED>;
    static std::atomic<uint64_t> asked{0};
    cudaError_t e = ask_shared_memory(kernel, sizeof(OwnShared), asked);
    if (e != cudaSuccess) return e;
    const int64_t ctas = std::min<int64_t>(int64_t(1) << g.shift, g.vocab);
    e = launch(kernel, dim3(static_cast<unsigned>(ctas)), kOwnThreads, sizeof(OwnShared), stream, g);
    if (e != cudaSuccess || pieces == 0) return e;
    return launch(novak_embedding_pieces_kernel<TYPE, GRAD, ALIGNED>, dim3(static_cast<unsigned>(pieces), static_cast<unsigned>(g.slices)),
                  kSumThreads, 0, stream, g);
}

}  // namespace

cudaError_t launch_embedding(const EmbedArgs &a, cudaStream_t stream)
{
    const bool aligned = wide(a.table, a.table_type, a.vocab) && wide(a.out, a.out_type, a.tokens) && a.cols % 8 == 0;
    LookArgs l{a, 0, 0};
    l.lanes = aligned ? power((a.cols + 7) / 8, 32) : 32;
    l.parts = static_cast<int>((a.cols + 8 * kLookGroups * l.lanes - 1) / (8 * kLookGroups * l.lanes));
    const int64_t ctas = (a.tokens * l.parts * l.lanes + kLookThreads - 1) / kLookThreads;
    const int which = a.table_type * 4 + a.out_type * 2 + aligned;
    const auto kernel = which == 0   ? novak_embedding_kernel<0, 0, false>
                        : which == 1 ? novak_embedding_kernel<0, 0, true>
                        : which == 2 ? novak_embedding_kernel<0, 1, false>
                        : which == 3 ? novak_embedding_kernel<0, 1, true>
                        : which == 4 ? novak_embedding_kernel<1, 0, false>
                        : which == 5 ? novak_embedding_kernel<1, 0, true>
                        : which == 6 ? novak_embedding_kernel<1, 1, false>
                                     : novak_embedding_kernel<1, 1, true>;
    return launch(kernel, dim3(static_cast<unsigned>(ctas)), kLookThreads, 0, stream, l);
}

size_t embedding_grad_bytes(int64_t tokens, int64_t, int64_t cols) { return layout_of(tokens, cols).bytes; }

cudaError_t launch_embedding_grad(const EmbedGradArgs &a, cudaStream_t stream)
{
    const GradLayout l = layout_of(a.tokens, a.cols);
    uint8_t *base = static_cast<uint8_t *>(a.work);
    GradArgs g{a, 8, l.pieces ? kPiece : INT_MAX, 0, l.slices, 0, reinterpret_cast<int *>(base + l.list), reinterpret_cast<Segment *>(base + l.order),
               reinterpret_cast<int *>(base + l.counts), reinterpret_cast<int *>(base + l.valid), reinterpret_cast<float *>(base + l.partial)};
    while ((a.vocab >> g.shift) >= kOwnRows) ++g.shift;
    g.lanes = power((a.cols + 7) / 8, 32);
    g.group = std::max(power((std::min<int64_t>(a.cols, kSlice) + 7) / 8, kSlice / 8), 32);
    const bool aligned = (a.tokens == 0 || wide(a.dout, a.type, a.tokens)) && wide(a.dtable, a.grad_type, a.vocab) && a.cols % 8 == 0;
    const int which = a.type * 4 + a.grad_type * 2 + aligned;
    return which == 0   ? launch_grad<0, 0, false>(g, l.pieces, stream)
           : which == 1 ? launch_grad<0, 0, true>(g, l.pieces, stream)
           : which == 2 ? launch_grad<0, 1, false>(g, l.pieces, stream)
           : which == 3 ? launch_grad<0, 1, true>(g, l.pieces, stream)
           : which == 4 ? launch_grad<1, 0, false>(g, l.pieces, stream)
           : which == 5 ? launch_grad<1, 0, true>(g, l.pieces, stream)
           : which == 6 ? launch_grad<1, 1, false>(g, l.pieces, stream)
                        : launch_grad<1, 1, true>(g, l.pieces, stream);
}

}  // namespace novak
