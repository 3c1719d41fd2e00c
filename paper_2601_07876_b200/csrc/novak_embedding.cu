// Token embedding, out[t] = scale table[ids[t]], and its gradient, the sum of dout's rows
// over the tokens of an id.
//
// Looking up is reading and writing rows; what bounds it is HBM (16384 of 50000 x 768 fp32 to bf16: 8.7 us,
// 7.8 at the copy rate), and for few tokens latency, so that long rows are cut among warps.
//
// The gradient of a whole table is mostly zeros to be written; the rest is to bring each id's
// tokens together in an order that goes by their places alone.  Two kernels.
// The first one orders the tokens.  No sort of all ids by digits: ids are dealt out by their low bits
// to some hundred CTAs (words of like frequency have like numbers; so they go to different ones),
// and each cluster of eight looks through all ids, an eighth each, and passes on to each other
// what is whose.  A CTA counts its rows' tokens and those of the CTAs before it, which says where its
// tokens lie in the order of all, and puts them there, row by row.
// The second one is one pass over dout and one over the table.  Warps have a few rows of 256 columns:
// zeros where there are no tokens, the sum of up to 16.  The order of all tokens is cut into pieces of 16
// besides, and those of longer rows have a CTA each; the last one of a row's pieces to be done adds
// their sums up in order.  So no word is too frequent.  (16384 tokens, some words frequent, 50000 x 768 bf16 to fp32:
// 47 us, 13 of them the first kernel's; 27.7 at the copy rate.)
// Of few tokens there is one kernel: every CTA looks through the ids for those of its own rows.
// (Zeros and sums in the first kernel, once it knows its rows: 58 to 77 us for 16384 tokens of 50000 x 768,
// since its shared memory leaves room for too few warps to hide what loads wait for.)
#include <algorithm>
#include <climits>

#include "novak_ops.cuh"
#include "novak_tcgen05.cuh"

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
        put_eight<ALIGNED>(out + i * a.lanes * 8, e, n[i]);
    }
}

// ---- the gradient --------------------------------------------------------------------
constexpr int kOwnThreads = 512, kOwnRows = 4096;       // rows of the table per CTA at most
constexpr int kCluster = 8;                             // CTAs that look through the ids together (each all of them: 33 MB out of L2, 8 us)
constexpr int kList = 4096, kBitWords = 4 * kOwnThreads;        // tokens that a CTA keeps in shared memory; words of its bit map
constexpr int kBits = 32 * kBitWords;                   // tokens in all that it has a bit for
constexpr int kPiece = 16;                              // tokens in a piece; rows of more go by pieces
constexpr int kSlice = 1024, kSumThreads = 256, kSumWarps = kSumThreads / 32;   // columns of a piece's CTA
// Tokens that one kernel alone does: 197 of 1003 x 768 fp32 3.9 us, 6.8 where some words are frequent, 10.4 where all
// are the same; two kernels with 513 7.8, 15.9, 20.3.  With 512 it would be 4.2, 12.4, and 29.7 (one CTA's sums).
constexpr int kFew = 256;
__host__ __device__ constexpr int64_t padded(int64_t cols) { return (cols + 3) / 4 * 4; }      // a piece's sums, in 16 bytes
constexpr int kMostRows = 16;                           // rows of a group of lanes in the second kernel

struct Place {              // of a token in the order of all; row < 0: its row is not summed by pieces
    int row, start, count, token;
};

struct GradArgs : EmbedGradArgs {
    int shift, fold;        // CTA p has the ids whose `shift` bits above the low `fold` ones are p
    int lanes;              // of a row, of 8 columns each
    int64_t steps;          // of that many columns
    int each;               // rows of a group of them, a power of two, up to kMostRows and `lanes`
    int slices, group;      // of kSlice columns; threads per token there
    int64_t pieces;         // CTAs of the second kernel that sum them
    bool few;               // and there is no first one
    void *list;             // for CTAs that have more than kList tokens: tokens; or of more than kBits in all int2, rows of the CTA and tokens
    Place *order;
    int2 *rows;             // of the table: how many tokens a row has, and where they are in that order; a single one itself
    int *counts;            // [piece][slice]: sums that are done, where a row begins in that piece
    int *valid;             // tokens in all
    float *partial;         // [piece][2][cols, padded]: of a row that began before, of one that begins here
};

// Sums over the CTA in the order of threads: those before this one, and all.
template <int THREADS> __device__ __forceinline__ int scan(int x, int *scratch, int &all)
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
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const int y = scratch[w];
        if (w < warp) before += y;
        all += y;
    }
    return before + s - x;
}

// Adds the lanes that are `mine` to counters[row]; the place of each.  Lanes of the first one's
// row go together (a word may be on all of them), the others by themselves.
__device__ __forceinline__ int count_rows(bool mine, int row, int *counters)
{
    const unsigned there = __ballot_sync(0xffffffffu, mine);
    if (there == 0) return 0;
    const int lane = threadIdx.x & 31, leader = __ffs(static_cast<int>(there)) - 1, of = __shfl_sync(0xffffffffu, row, leader);
    const bool together = mine && row == of;
    const unsigned same = __ballot_sync(0xffffffffu, together);
    int place = 0;
    if (lane == leader || (mine && !together)) place = atomicAdd(counters + row, together ? __popc(same) : 1);
    const int base = __shfl_sync(0xffffffffu, place, leader);
    return together ? base + __popc(same & ((1u << lane) - 1)) : place;
}

// In another CTA's shared memory (addresses from at_rank).
__device__ __forceinline__ uint32_t atomic_add_at(uint32_t addr, uint32_t x)
{
    uint32_t r;
    asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(r) : "r"(addr), "r"(x) : "memory");
    return r;
}
__device__ __forceinline__ void store_at(uint32_t addr, int x) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(x) : "memory"); }
__device__ __forceinline__ void store_at(uint32_t addr, uint16_t x) { asm volatile("st.shared::cluster.u16 [%0], %1;" ::"r"(addr), "h"(x) : "memory"); }

constexpr int kFetched = 8;                             // ids of a thread on their way, where a CTA looks through all of them
static_assert(kOwnRows <= kList, "a place for each row");

// (98604 bytes.  1 KB more, and two CTAs no longer fit the split of an SM's memory that the second kernel takes as well:
// setting it anew costs 2 us a call.)
struct OwnShared {
    int counts[kOwnRows], starts[kOwnRows];
    int found[kList], list[kList];              // tokens as they were found (or, of more, where each row's next one goes); row by row
    uint16_t found_row[kList];
    __align__(16) uint32_t bits[kBitWords];
    uint16_t few[kOwnRows], many[kOwnRows];     // rows of 1 to 16 tokens, and of more
    int passed[kCluster];                       // tokens that this CTA found, by whose they are
    int before[kCluster], valid[kCluster];      // of each CTA's share of the ids: those of CTAs before this one; all
    int sums[2][kOwnThreads / 32], scratch[kOwnThreads / 32];
    int n, n_few, n_many;
};

// How ids are dealt out, as a CTA sees it: blocks of 2^fold rows: own, own + 2^shift, ...; some of the last one's may be
// beyond the table.
struct Dealt {
    const int64_t own, low;
    const int fold, above, inside, rows;
    __device__ __forceinline__ explicit Dealt(const GradArgs &a)
        : own(blockIdx.x), low((int64_t(1) << a.shift) - 1), fold(a.fold), above(a.fold + a.shift), inside((1 << a.fold) - 1),
          rows(static_cast<int>(max((((a.vocab + inside) >> fold) - own + low) >> a.shift, static_cast<int64_t>(0)) << fold))
    {
    }
    __device__ __forceinline__ int row_of(int64_t id) const { return static_cast<int>(id >> above << fold | (id & inside)); }
    __device__ __forceinline__ int64_t id_of(int row) const { return static_cast<int64_t>(row >> fold) << above | own << fold | (row & inside); }
    __device__ __forceinline__ uint32_t owner(uint32_t id) const { return id >> fold & static_cast<uint32_t>(low); }
};

// The ids from t0 on, N a thread (what is none: the largest number).
template <int N> __device__ __forceinline__ void fetch_ids(const GradArgs &a, int64_t t0, uint32_t (&id)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t t = t0 + k * kOwnThreads + threadIdx.x, x = t < a.tokens ? id_at(a.ids, a.id_type, t) : -1;
        id[k] = x >= 0 && x < a.vocab ? static_cast<uint32_t>(x) : ~0u;
    }
}

// Places for a warp's tokens among those of the CTAs `whose` they are: kList for who has none.
__device__ __forceinline__ uint32_t places(bool ours, uint32_t whose, OwnShared &sh)
{
    const unsigned all = __ballot_sync(0xffffffffu, ours);
    if (__popc(all) <= 4) {
        if (!ours) return kList;
        atomicAdd(&sh.passed[whose], 1);
        return atomic_add_at(at_rank(smem_addr(&sh.n), whose), 1);
    }
    // some word is frequent: one addition for all of a CTA's
    const int lane = threadIdx.x & 31;
    uint32_t at = kList;
    for (unsigned left = all; left;) {
        const int leader = __ffs(static_cast<int>(left)) - 1;
        const uint32_t of = __shfl_sync(0xffffffffu, whose, leader);
        const unsigned same = __ballot_sync(0xffffffffu, ours && whose == of);
        left &= ~same;
        uint32_t base = 0;
        if (lane == leader) {
            atomicAdd(&sh.passed[of], __popc(same));
            base = atomic_add_at(at_rank(smem_addr(&sh.n), of), __popc(same));
        }
        base = __shfl_sync(0xffffffffu, base, leader);
        if (same >> lane & 1) at = base + __popc(same & ((1u << lane) - 1));
    }
    return at;
}

// All ids, for this CTA's tokens in order, whatever their number, and how many each of its rows has.
__device__ __forceinline__ void list_in_order(const GradArgs &a, const Dealt &deal, OwnShared &sh, int2 *list)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kSums = kFetched * kOwnThreads / 32, kEach = kSums / 32;
    static_assert(kEach == 4 && 2 * kSums <= kBitWords, "an int4; two of them in the map's place");
    int *const found_now = reinterpret_cast<int *>(sh.bits);       // tokens of 32 ids each
    uint32_t id[kFetched], next[kFetched];
    fetch_ids(a, 0, id);
    int done = 0, turn = 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kFetched * kOwnThreads, turn ^= 1) {
        fetch_ids(a, t0 + kFetched * kOwnThreads, next);
        unsigned mine[kFetched];
#pragma unroll
        for (int k = 0; k < kFetched; ++k) {
            mine[k] = __ballot_sync(0xffffffffu, id[k] != ~0u && deal.owner(id[k]) == deal.own);
            if (lane == 0) found_now[turn * kSums + k * (kOwnThreads / 32) + warp] = __popc(mine[k]);
        }
        __syncthreads();            // (two of them by turns: one barrier is enough)
        // where each 32 ids' tokens go: four sums of them a lane
        const int4 sums = *reinterpret_cast<const int4 *>(found_now + turn * kSums + lane * kEach);
        const int sum = sums.x + sums.y + sums.z + sums.w;
        int to_here = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, to_here, d);
            if (lane >= d) to_here += y;
        }
#pragma unroll
        for (int k = 0; k < kFetched; ++k) {
            if (mine[k] != 0) {             // (most often none is, and all of this is the cost of a pass over all ids)
                const int which = k * (kOwnThreads / 32) + warp, i = which % kEach;
                const int in_lane = (i > 0 ? sums.x : 0) + (i > 1 ? sums.y : 0) + (i > 2 ? sums.z : 0);
                const int at = __shfl_sync(0xffffffffu, to_here - sum + in_lane, which / kEach), row = deal.row_of(id[k]);
                const bool it = mine[k] >> lane & 1;
                if (it) list[done + at + __popc(mine[k] & ((1u << lane) - 1))] = make_int2(row, static_cast<int>(t0 + k * kOwnThreads + threadIdx.x));
                count_rows(it, row, sh.counts);
            }
            id[k] = next[k];
        }
        done += __shfl_sync(0xffffffffu, to_here, 31);
    }
}

// The order of a list that is in order: each warp has some of the rows, and goes through all of the list.
__device__ __forceinline__ void order_list(const GradArgs &a, const Dealt &deal, OwnShared &sh, const int2 *list, int before, int n)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kOwnThreads / 32;
    for (int i = threadIdx.x; i < deal.rows; i += kOwnThreads) sh.found[i] = sh.starts[i];
    __syncthreads();
    const auto put = [&](int row, int token, int place, int count, int start, unsigned same) {
        const int id = static_cast<int>(deal.id_of(row)), at = before + place + __popc(same & ((1u << lane) - 1));
        if (count == 1) a.rows[id] = make_int2(token, 1);
        a.order[at] = count > kPiece ? Place{id, before + start, count, token} : Place{-1, 0, 0, token};
    };
    // (a word may be on most of them: the place of one row's next token is at hand, the others' are in shared memory)
    int held = -1, held_place = 0, held_count = 0, held_start = 0;
    for (int i0 = 0; i0 < n; i0 += 32 * kFetched) {
        int2 x[kFetched];           // (no row's number is negative)
#pragma unroll
        for (int k = 0; k < kFetched; ++k) x[k] = i0 + k * 32 + lane < n ? list[i0 + k * 32 + lane] : make_int2(-1, 0);
#pragma unroll
        for (int k = 0; k < kFetched; ++k) {
            const int row = x[k].x;
            const bool mine = row >= 0 && row % kWarps == warp;
            const unsigned of_held = __ballot_sync(0xffffffffu, mine && row == held);
            if (mine && row == held) put(row, x[k].y, held_place, held_count, held_start, of_held);
            held_place += __popc(of_held);
            // the others, row by row
            for (unsigned left = __ballot_sync(0xffffffffu, mine) & ~of_held; left;) {
                const int of = __shfl_sync(0xffffffffu, row, __ffs(static_cast<int>(left)) - 1);
                const unsigned same = __ballot_sync(0xffffffffu, row == of);
                left &= ~same;
                const int place = sh.found[of], next = place + __popc(same), count = sh.counts[of], start = sh.starts[of];
                if (row == of) put(row, x[k].y, place, count, start, same);
                __syncwarp();
                const bool hold = __popc(same) > __popc(of_held);
                if (lane == 0) {
                    sh.found[of] = next;
                    if (hold && held >= 0) sh.found[held] = held_place;
                }
                __syncwarp();
                if (hold) {
                    held = of;
                    held_place = next;
                    held_count = count;
                    held_start = start;
                }
            }
        }
    }
    for (int k = 0; k < sh.n_many; ++k)
        for (int i = threadIdx.x; i < a.slices; i += kOwnThreads) a.counts[static_cast<int64_t>((before + sh.starts[sh.many[k]]) / kPiece) * a.slices + i] = 0;
}

// The rows of many tokens by comparing each with all of its row, a warp 32 of them at a time.
__device__ __forceinline__ void order_by_comparing(const GradArgs &a, const Dealt &deal, const OwnShared &sh, int before)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int unit = 0;
    for (int k = 0; k < sh.n_many; ++k) {
        const int row = sh.many[k], count = sh.counts[row], first = sh.starts[row] - count;
        for (int i = 0; i < count; i += 32, ++unit) {
            if (unit % (kOwnThreads / 32) != warp) continue;
            const int x = i + lane < count ? sh.list[first + i + lane] : INT_MAX;
            int place = 0;
#pragma unroll 8
            for (int j = 0; j < count; ++j) place += sh.list[first + j] < x;
            if (i + lane < count) a.order[before + first + place] = Place{static_cast<int>(deal.id_of(row)), before + first, count, x};
        }
        for (int i = threadIdx.x; i < a.slices; i += kOwnThreads) a.counts[static_cast<int64_t>((before + first) / kPiece) * a.slices + i] = 0;
    }
}

// LONG: of more tokens in all than the map has bits for.  A map a row for each 65536 of them would cost their number times
// the rows' (1048576 tokens of 50000 words alike, 16 columns: 4.7 ms, this way 1.3; 4194304 of one word 114 and 24).
template <bool LONG>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kOwnThreads, 2) novak_embedding_order_kernel(GradArgs a)
{
    extern __shared__ uint8_t raw_shared[];
    OwnShared &sh = *reinterpret_cast<OwnShared *>(raw_shared);
    const Dealt deal(a);
    const int64_t own = deal.own;
    const int rows = deal.rows;
    const auto id_of = [&](int row) { return deal.id_of(row); };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < rows; i += kOwnThreads) sh.counts[i] = 0;
    if (threadIdx.x < kCluster) sh.passed[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n = sh.n_few = sh.n_many = 0;
    cluster_sync();
    start();

    // ---- this CTA's share of the ids: whose they are, and how many belong to CTAs before this cluster
    constexpr int kAhead = 4;
    const uint32_t rank = cluster_rank(), cluster0 = static_cast<uint32_t>(own) - rank;
    {
        int before = 0, valid = 0;
        for (int64_t t0 = rank * kAhead * kOwnThreads; t0 < a.tokens; t0 += kCluster * kAhead * kOwnThreads) {
            uint32_t id[kAhead];
            fetch_ids(a, t0, id);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const uint32_t whose = deal.owner(id[k]) - cluster0;
                uint32_t at;
                if constexpr (LONG) {
                    const bool there = id[k] != ~0u, ours = there && whose < kCluster;
                    valid += there;
                    before += there && deal.owner(id[k]) < cluster0;
                    at = places(ours, whose, sh);
                } else {
                    if (id[k] == ~0u) continue;
                    ++valid;
                    before += deal.owner(id[k]) < cluster0;
                    if (whose >= kCluster) continue;
                    atomicAdd(&sh.passed[whose], 1);
                    at = atomic_add_at(at_rank(smem_addr(&sh.n), whose), 1);
                }
                if (at < kList) {
                    store_at(at_rank(smem_addr(&sh.found[at]), whose), static_cast<int>(t0 + k * kOwnThreads + threadIdx.x));
                    store_at(at_rank(smem_addr(&sh.found_row[at]), whose), static_cast<uint16_t>(deal.row_of(id[k])));
                }
            }
        }
        before = __reduce_add_sync(0xffffffffu, before);
        valid = __reduce_add_sync(0xffffffffu, valid);
        if (lane == 0) {
            sh.sums[0][warp] = before;
            sh.sums[1][warp] = valid;
        }
        __syncthreads();
        if (threadIdx.x < kCluster) {
            before = valid = 0;
            for (int w = 0; w < kOwnThreads / 32; ++w) {
                before += sh.sums[0][w];
                valid += sh.sums[1][w];
            }
            for (int r = 0; r < static_cast<int>(threadIdx.x); ++r) before += sh.passed[r];
            store_at(at_rank(smem_addr(&sh.before[rank]), threadIdx.x), before);
            store_at(at_rank(smem_addr(&sh.valid[rank]), threadIdx.x), valid);
        }
    }
    cluster_sync();             // (from here on nobody looks into another CTA)
    int before = 0;
    for (int r = 0; r < kCluster; ++r) before += sh.before[r];
    if (own == 0 && threadIdx.x == 0) {
        int valid = 0;
        for (int r = 0; r < kCluster; ++r) valid += sh.valid[r];
        *a.valid = valid;
    }
    const int n = sh.n;
    if (n <= kList) {
        for (int i = warp * 32; i < n; i += kOwnThreads) count_rows(i + lane < n, i + lane < n ? sh.found_row[i + lane] : 0, sh.counts);
    } else if constexpr (LONG) {
        list_in_order(a, deal, sh, static_cast<int2 *>(a.list) + before);
    } else {
        for (int64_t t0 = 0; t0 < a.tokens; t0 += kFetched * kOwnThreads) {
            uint32_t id[kFetched];
            fetch_ids(a, t0, id);
#pragma unroll
            for (int k = 0; k < kFetched; ++k) count_rows(id[k] != ~0u && deal.owner(id[k]) == own, deal.row_of(id[k]), sh.counts);
        }
    }
    __syncthreads();

    // ---- where each row's tokens begin
    {
        constexpr int kEach = kOwnRows / kOwnThreads;
        const int first = threadIdx.x * kEach;
        int sum = 0, all;
        if (first < rows)
            for (int i = first; i < min(first + kEach, rows); ++i) sum += sh.counts[i];
        int at = scan<kOwnThreads>(sum, sh.scratch, all);
        if (first < rows)
            for (int i = first; i < min(first + kEach, rows); ++i) {
                const int count = sh.counts[i];
                sh.starts[i] = at;
                if (count > 0 && count <= kPiece) sh.few[atomicAdd(&sh.n_few, 1)] = static_cast<uint16_t>(i);
                if (count > kPiece) sh.many[atomicAdd(&sh.n_many, 1)] = static_cast<uint16_t>(i);
                at += count;
            }
    }
    __syncthreads();
    for (int row = threadIdx.x; row < rows; row += kOwnThreads)
        if (id_of(row) < a.vocab && sh.counts[row] != 1) a.rows[id_of(row)] = make_int2(before + sh.starts[row], sh.counts[row]);
    __syncthreads();

    // ---- the tokens, row by row: put there in any order (starts go up to the ends) ...
    int *const list = LONG || n <= kList ? sh.list : static_cast<int *>(a.list) + before;
    if (n <= kList) {
        for (int i = warp * 32; i < n; i += kOwnThreads) {
            const bool in = i + lane < n;
            const int place = count_rows(in, in ? sh.found_row[i + lane] : 0, sh.starts);
            if (in) list[place] = sh.found[i + lane];
        }
    } else if constexpr (LONG) {
        order_list(a, deal, sh, static_cast<const int2 *>(a.list) + before, before, n);
        return;
    } else {
        for (int64_t t0 = 0; t0 < a.tokens; t0 += kFetched * kOwnThreads) {
            uint32_t id[kFetched];
            fetch_ids(a, t0, id);
#pragma unroll
            for (int k = 0; k < kFetched; ++k) {
                const bool mine = id[k] != ~0u && deal.owner(id[k]) == own;
                if (!__any_sync(0xffffffffu, mine)) continue;
                const int place = count_rows(mine, deal.row_of(id[k]), sh.starts);
                if (mine) list[place] = static_cast<int>(t0 + k * kOwnThreads + threadIdx.x);
            }
        }
    }
    __syncthreads();

    // ... and then in order.  Of few tokens a lane has one each: its place is the number of tokens before it.
    const int n_few = sh.n_few;
    for (int i = warp; i < n_few; i += kOwnThreads / 32) {
        const int row = sh.few[i], count = sh.counts[row], first = sh.starts[row] - count;
        if (count == 1 && lane == 0) a.rows[id_of(row)] = make_int2(list[first], 1);
        const int x = lane < count ? list[first + lane] : INT_MAX;
        int place = 0;
        for (int j = 0; j < count; ++j) place += __shfl_sync(0xffffffffu, x, j) < x;
        if (lane < count) a.order[before + first + place] = Place{-1, 0, 0, x};
    }
    if constexpr (LONG) {
        order_by_comparing(a, deal, sh, before);
    } else {
        // Many: the tokens as bits of a map.
        for (int k = 0; k < sh.n_many; ++k) {
            const int row = sh.many[k], count = sh.counts[row], first = sh.starts[row] - count;
            __syncthreads();
            for (int i = threadIdx.x; i < kBitWords; i += kOwnThreads) sh.bits[i] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < count; i += kOwnThreads) {
                const int t = list[first + i];
                atomicOr(&sh.bits[t >> 5], 1u << (t & 31));
            }
            __syncthreads();
            constexpr int kEach = kBitWords / kOwnThreads;
            int bits = 0, all;
            for (int i = 0; i < kEach; ++i) bits += __popc(sh.bits[threadIdx.x * kEach + i]);
            int at = scan<kOwnThreads>(bits, sh.scratch, all);
            for (int i = 0; i < kEach; ++i)
                for (uint32_t m = sh.bits[threadIdx.x * kEach + i]; m; m &= m - 1, ++at) {
                    const int t = (threadIdx.x * kEach + i) * 32 + __ffs(static_cast<int>(m)) - 1;
                    a.order[before + first + at] = Place{static_cast<int>(id_of(row)), before + first, count, t};
                }
            for (int i = threadIdx.x; i < a.slices; i += kOwnThreads) a.counts[static_cast<int64_t>((before + first) / kPiece) * a.slices + i] = 0;
        }
    }
}

// Eight columns of the sum over `count` tokens.
template <int TYPE, bool ALIGNED, typename Token>
__device__ __forceinline__ void sum_tokens(const EmbedGradArgs &a, const Token &token, int count, int64_t col, int n, const void *begin,
                                           const void *end, F2 (&sum)[4])
{
    using T = typename Elem<TYPE>::T;
    constexpr int kAhead = TYPE == NOVAK_TYPE_BF16 && ALIGNED ? 8 : 4;
    const T *base = static_cast<const T *>(a.dout.ptr) + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = F2(0.0f);
    for (int j = 0; j < count; j += kAhead) {
        Fetch<TYPE, ALIGNED> raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            raw[k].zero();
            if (j + k < count) raw[k].load(base + token(j + k) * a.dout.stride, n, begin, end);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (j + k < count) {
                F2 v[4];
                raw[k].eight().get(v);
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
    put_eight<ALIGNED>(p, e, n);
}

// A piece of the order of all tokens, kSlice columns: of at most two rows, since each row here has more tokens than a
// piece has: one that began before, and one that begins here.
template <int TYPE, int GRAD, bool ALIGNED> __device__ __forceinline__ void sum_piece(const GradArgs &a, int piece, int slice)
{
    using G = typename Elem<GRAD>::T;
    using T = typename Elem<TYPE>::T;
    __shared__ __align__(16) float part[kSumThreads * 8];
    __shared__ Place first, second;
    __shared__ int begins;
    __shared__ bool last;
    __shared__ int tokens[kPiece];
    const int from = piece * kPiece;
    if (threadIdx.x < 32) {
        Place s{-1, 0, 0, 0};
        const int valid = *a.valid, at_most = static_cast<int>(min(a.tokens - from, static_cast<int64_t>(kPiece))), lane = threadIdx.x;
        if (lane < at_most) s = a.order[from + lane];           // (nothing there behind the valid ones)
        if (from + lane >= valid) s.row = -1;
        if (lane < kPiece) tokens[lane] = s.token;
        const unsigned m = __ballot_sync(0xffffffffu, s.row >= 0 && s.start == from + static_cast<int>(threadIdx.x));
        const int at = m ? __ffs(static_cast<int>(m)) - 1 : kPiece;
        if (threadIdx.x == 0) {
            begins = at;
            first = s;
        }
        if (static_cast<int>(threadIdx.x) == at) second = s;
    }
    static_assert(kPiece <= 32, "a warp looks at a piece");
    __syncthreads();
    const int group = a.group, subs = kSumThreads / group, sub = threadIdx.x / group, t = threadIdx.x % group;
    const int64_t col = static_cast<int64_t>(slice) * kSlice + t * 8;
    const int n = static_cast<int>(max(min(a.cols - col, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
    const void *begin = a.dout.ptr, *end = end_of(static_cast<const T *>(a.dout.ptr), a.dout.stride, a.tokens, a.cols);
    for (int kind = 0; kind < 2; ++kind) {
        const int at = kind ? begins : 0;
        if (kind ? begins == kPiece : first.row < 0 || begins == 0) continue;
        const Place seg = kind ? second : first;
        const int count = min(seg.start + seg.count - from, kPiece) - at;
        // this piece: every group of threads its share of the tokens, then the groups in order
        F2 sum[4];
        const int share = (count + subs - 1) / subs, begin_at = min(sub * share, count);
        sum_tokens<TYPE, ALIGNED>(a, [&](int k) { return tokens[at + begin_at + k]; }, min(share, count - begin_at), col, n, begin, end, sum);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2 *>(part + threadIdx.x * 8 + 2 * i) = make_float2(sum[i].lo(), sum[i].hi());
        __syncthreads();
        for (int c = threadIdx.x; c < group * 8; c += kSumThreads) {
            float x = 0.0f;
            for (int i = 0; i < subs; ++i) x += part[i * group * 8 + c];
            const int64_t out = static_cast<int64_t>(slice) * kSlice + c;
            if (out < a.cols) a.partial[(2 * static_cast<int64_t>(piece) + kind) * padded(a.cols) + out] = x;
        }
        // the last of the row's pieces to be done adds all of them up
        const int head = seg.start / kPiece, pieces = (seg.start + seg.count - 1) / kPiece - head + 1;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(a.counts + static_cast<int64_t>(head) * a.slices + slice, 1) + 1 == pieces;
        __syncthreads();
        if (!last) continue;
        __threadfence();
        // four columns a thread, a share of the pieces each, then the shares in order (16384 tokens of one row of 768: 181 us;
        // a column a thread and all of the pieces, 241; some words frequent: 46 and 51)
        const int quads = group * 2, shares = kSumThreads / quads, mine = threadIdx.x / quads, quad = threadIdx.x % quads;
        const int each = (pieces + shares - 1) / shares, end_at = min((mine + 1) * each, pieces);
        const int64_t out = static_cast<int64_t>(slice) * kSlice + quad * 4;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (out < a.cols) {
            const float *p = a.partial + 2 * static_cast<int64_t>(head) * padded(a.cols) + out;
#pragma unroll 8
            for (int i = mine * each; i < end_at; ++i) {        // (behind the first one: of a row that began before)
                const float4 y = __ldcg(reinterpret_cast<const float4 *>(p + (i == 0 ? 1 : 2 * static_cast<int64_t>(i)) * padded(a.cols)));
                x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            }
        }
        *reinterpret_cast<float4 *>(part + threadIdx.x * 4) = x;
        __syncthreads();
        if (mine == 0) {
            for (int i = 1; i < shares; ++i) {
                const float4 y = *reinterpret_cast<const float4 *>(part + (i * quads + quad) * 4);
                x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            }
            *reinterpret_cast<float4 *>(part + quad * 4) = x;
        }
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < group) {
            F2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = F2(part[threadIdx.x * 8 + 2 * i], part[threadIdx.x * 8 + 2 * i + 1]);
            G *p = static_cast<G *>(a.dtable.ptr) + static_cast<int64_t>(seg.row) * a.dtable.stride + col;
            put_sum<GRAD, ALIGNED>(a, p, n, v, a.dtable.ptr, end_of(static_cast<const G *>(a.dtable.ptr), a.dtable.stride, a.vocab, a.cols));
        }
        __syncthreads();
    }
}

// A group of lanes' rows from row0 on, eight columns a lane: zeros, and sums of up to kPiece tokens.  A lane knows
// of a row what `mine` says (see GradArgs::rows).
template <int TYPE, int GRAD, bool ALIGNED, typename Token>
__device__ __forceinline__ void write_rows(const GradArgs &a, int2 mine, int lanes, int64_t row0, int64_t col, const Token &token)
{
    using G = typename Elem<GRAD>::T;
    using T = typename Elem<TYPE>::T;
    const int lane = threadIdx.x % lanes, shift = threadIdx.x % 32 / lanes * lanes;
    const int n = static_cast<int>(max(min(a.cols - col, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
    const void *begin = a.dout.ptr, *end = end_of(static_cast<const T *>(a.dout.ptr), a.dout.stride, a.tokens, a.cols);
    const void *out_begin = a.dtable.ptr, *out_end = end_of(static_cast<const G *>(a.dtable.ptr), a.dtable.stride, a.vocab, a.cols);
    const unsigned group = lanes == 32 ? ~0u : ((1u << lanes) - 1) << shift;
    G *p = static_cast<G *>(a.dtable.ptr) + row0 * a.dtable.stride + col;
    unsigned none = (__ballot_sync(0xffffffffu, mine.y == 0 && lane < a.each) & group) >> shift;
    unsigned one = (__ballot_sync(0xffffffffu, mine.y == 1) & group) >> shift;
    unsigned some = (__ballot_sync(0xffffffffu, mine.y > 1 && mine.y <= kPiece) & group) >> shift;
    if (!a.add)
        for (; none; none &= none - 1) {
            G *row = p + (__ffs(static_cast<int>(none)) - 1) * a.dtable.stride;
            if constexpr (ALIGNED && GRAD == NOVAK_TYPE_F32) {
                // (neighbouring lanes neighbouring pieces: with 32 bytes each, in two stores, 40 us instead of 24)
                float4 *piece = reinterpret_cast<float4 *>(row - lane * 8) + lane;
                const int64_t left = (a.cols - (col - lane * 8)) / 4 - lane;
                if (left > 0) piece[0] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (left > lanes) piece[lanes] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            } else {
                Eight<GRAD> e;
                e.zero();
                store_eight<ALIGNED>(row, e, n);
            }
        }
    // rows of one token (most): several on their way
    constexpr int kRows = TYPE == NOVAK_TYPE_BF16 && ALIGNED ? 4 : 2;
    while (__any_sync(0xffffffffu, one != 0)) {
        Fetch<TYPE, ALIGNED> raw[kRows];
        int at[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k, one &= one - 1) {
            at[k] = __ffs(static_cast<int>(one)) - 1;           // -1: none
            const int token = __shfl_sync(0xffffffffu, mine.x, max(at[k], 0), lanes);
            raw[k].zero();
            if (at[k] >= 0) raw[k].load(static_cast<const T *>(a.dout.ptr) + token * a.dout.stride + col, n, begin, end);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (at[k] < 0 || (ALIGNED && n == 0)) continue;
            F2 sum[4];
            raw[k].eight().get(sum);
            put_sum<GRAD, ALIGNED>(a, p + at[k] * a.dtable.stride, n, sum, out_begin, out_end);
        }
    }
    for (; __any_sync(0xffffffffu, some != 0); some &= some - 1) {
        const int i = some ? __ffs(static_cast<int>(some)) - 1 : 0;
        const int first = __shfl_sync(0xffffffffu, mine.x, i, lanes), count = __shfl_sync(0xffffffffu, mine.y, i, lanes);
        if (some == 0 || (ALIGNED && n == 0)) continue;
        F2 sum[4];
        sum_tokens<TYPE, ALIGNED>(a, [&](int k) { return token(first + k); }, count, col, n, begin, end, sum);
        put_sum<GRAD, ALIGNED>(a, p + i * a.dtable.stride, n, sum, out_begin, out_end);
    }
}

template <int TYPE, int GRAD, bool ALIGNED>
__global__ void __launch_bounds__(kSumThreads, ALIGNED ? 4 : 3) novak_embedding_grad_kernel(GradArgs a)
{
    start();
    // Pieces first, since they take long, but by turns with the others: they wait more than they move.
    const int64_t pieces = a.pieces * a.slices, rest = gridDim.x - pieces, both = 2 * min(pieces, rest), b = blockIdx.x;
    const bool is_piece = b < both ? b % 2 == 0 : pieces > rest;
    const int64_t index = b < both ? b / 2 : b - both / 2;
    if (is_piece) {
        const int piece = static_cast<int>(index / a.slices);
        sum_piece<TYPE, GRAD, ALIGNED>(a, piece, static_cast<int>(index - static_cast<int64_t>(piece) * a.slices));
        return;
    }
    const int lanes = ALIGNED ? a.lanes : 32, lane = threadIdx.x % lanes;
    const int64_t item = index * kSumWarps + threadIdx.x / 32;
    const int64_t block = item <= INT_MAX && a.steps <= INT_MAX ? static_cast<unsigned>(item) / static_cast<unsigned>(a.steps) : item / a.steps;
    const int64_t col = ((item - block * a.steps) * lanes + lane) * 8;
    const int64_t row0 = (block * (32 / lanes) + threadIdx.x % 32 / lanes) * a.each;
    // rows beyond the table are nobody's
    int2 mine = make_int2(0, INT_MAX);
    if (lane < a.each && row0 + lane < a.vocab) mine = a.rows[row0 + lane];
    write_rows<TYPE, GRAD, ALIGNED>(a, mine, lanes, row0, col, [&](int k) { return a.order[k].token; });
}

// Few tokens: one kernel, each of whose CTAs looks through all ids for those of its rows, kSumWarps times a warp's.
template <int TYPE, int GRAD, bool ALIGNED>
__global__ void __launch_bounds__(kSumThreads, ALIGNED ? 4 : 3) novak_embedding_few_grad_kernel(GradArgs a)
{
    using G = typename Elem<GRAD>::T;
    using T = typename Elem<TYPE>::T;
    __shared__ int found[kFew], order[kFew], scratch[kSumWarps];
    __shared__ __align__(16) uint16_t found_row[kFew + 8];
    __shared__ uint16_t many[kFew / kPiece];
    __shared__ int2 rows[kSumThreads];
    __shared__ int n_many;
    __shared__ __align__(16) float part[kSumThreads * 8];
    const int lanes = ALIGNED ? a.lanes : 32, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
    const int64_t block = blockIdx.x / a.steps, col = ((blockIdx.x - block * a.steps) * lanes + lane) * 8;
    const int height = kSumThreads / lanes * a.each;        // (at most kSumThreads)
    const int64_t row0 = block * height;
    if (threadIdx.x == 0) n_many = 0;
    start();

    // the tokens whose rows are here, in order
    constexpr int kEach = kFew / kSumThreads;
    int64_t id[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int t = threadIdx.x * kEach + i;
        id[i] = t < a.tokens ? id_at(a.ids, a.id_type, t) : -1;
    }
    const int64_t here = min(static_cast<int64_t>(height), a.vocab - row0);
    int count = 0, n;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        id[i] = id[i] >= row0 && id[i] - row0 < here ? id[i] - row0 : -1;
        count += id[i] >= 0;
    }
    int at = scan<kSumThreads>(count, scratch, n);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (id[i] >= 0) {
            found[at] = threadIdx.x * kEach + i;
            found_row[at++] = static_cast<uint16_t>(id[i]);
        }
    if (threadIdx.x < 8) found_row[n + threadIdx.x] = 0xffff;
    rows[threadIdx.x] = make_int2(0, 0);
    __syncthreads();
    // each token: how many of its row there are, and how many of them before it
    int before[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = k * kSumThreads + threadIdx.x;
        if (i >= n) continue;
        const int row = found_row[i];
        int of_row = 0, place = 0;
        for (int j = 0; j < n; j += 8) {
            const uint4 w = *reinterpret_cast<const uint4 *>(found_row + j);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const bool same = static_cast<int>(u[m / 2] >> m % 2 * 16 & 0xffffu) == row;
                of_row += same;
                place += same && j + m < i;
            }
        }
        before[k] = place;
        if (place == 0) rows[row].y = of_row;
    }
    __syncthreads();
    count = rows[threadIdx.x].y;
    int all;
    at = scan<kSumThreads>(count, scratch, all);
    if (count > kPiece) many[atomicAdd(&n_many, 1)] = static_cast<uint16_t>(threadIdx.x);
    rows[threadIdx.x].x = at;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = k * kSumThreads + threadIdx.x;
        if (i < n) order[rows[found_row[i]].x + before[k]] = found[i];
    }
    __syncthreads();
    if (count == 1) rows[threadIdx.x].x = order[at];
    __syncthreads();
    int2 mine = make_int2(0, INT_MAX);
    if (lane < a.each && group * a.each + lane < here) mine = rows[group * a.each + lane];
    write_rows<TYPE, GRAD, ALIGNED>(a, mine, lanes, row0 + group * a.each, col, [&](int k) { return order[k]; });

    // rows of more: every group of lanes its share of the tokens, then the groups in order
    const int n_columns = static_cast<int>(max(min(a.cols - col, static_cast<int64_t>(8)), static_cast<int64_t>(0)));
    const int groups = kSumThreads / lanes;
    for (int m = 0; m < n_many; ++m) {
        const int row = many[m], share = (rows[row].y + groups - 1) / groups, first = min(group * share, rows[row].y);
        F2 sum[4];
        const int *tokens = order + rows[row].x + first;
        sum_tokens<TYPE, ALIGNED>(a, [&](int k) { return tokens[k]; }, min(share, rows[row].y - first), col, n_columns, a.dout.ptr,
                                  end_of(static_cast<const T *>(a.dout.ptr), a.dout.stride, a.tokens, a.cols), sum);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2 *>(part + threadIdx.x * 8 + 2 * i) = make_float2(sum[i].lo(), sum[i].hi());
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = F2(0.0f);
            for (int k = 0; k < groups; ++k) {
                const float *p = part + (k * lanes + lane) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = sum[i] + F2(p[2 * i], p[2 * i + 1]);
            }
            G *p = static_cast<G *>(a.dtable.ptr) + (row0 + row) * a.dtable.stride + col;
            put_sum<GRAD, ALIGNED>(a, p, n_columns, sum, a.dtable.ptr, end_of(static_cast<const G *>(a.dtable.ptr), a.dtable.stride, a.vocab, a.cols));
        }
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
    size_t list, order, rows, counts, valid, partial, bytes;
};

GradLayout layout_of(int64_t tokens, int64_t vocab, int64_t cols)
{
    GradLayout l{};
    l.pieces = tokens > kPiece ? (tokens + kPiece - 1) / kPiece : 0;        // (fewer tokens are no long row's)
    l.slices = static_cast<int>((cols + kSlice - 1) / kSlice);
    l.list = 0;
    l.order = l.list + round_up((tokens > kBits ? tokens * sizeof(int2) : tokens > kList ? tokens * sizeof(int) : 0));
    l.rows = l.order + round_up(tokens * sizeof(Place));
    l.counts = l.rows + round_up(vocab * sizeof(int2));
    l.valid = l.counts + round_up(l.pieces * l.slices * sizeof(int));
    l.partial = l.valid + round_up(sizeof(int));
    l.bytes = l.partial + round_up(2 * l.pieces * padded(cols) * sizeof(float));
    return l;
}

template <int TYPE, int GRAD, bool ALIGNED> cudaError_t launch_grad(const GradArgs &g, cudaStream_t stream)
{
    const int lanes = ALIGNED ? g.lanes : 32, rows = g.each * (32 / lanes);
    if (g.few) {
        const int64_t blocks = (g.vocab + rows * kSumWarps - 1) / (rows * kSumWarps);
        return launch(novak_embedding_few_grad_kernel<TYPE, GRAD, ALIGNED>, dim3(static_cast<unsigned>(blocks * g.steps)), kSumThreads, 0, stream, g);
    }
    const int64_t items = (g.vocab + rows - 1) / rows * g.steps, ctas = g.pieces * g.slices + (items + kSumWarps - 1) / kSumWarps;
    return launch(novak_embedding_grad_kernel<TYPE, GRAD, ALIGNED>, dim3(static_cast<unsigned>(ctas)), kSumThreads, 0, stream, g);
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

size_t embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t cols) { return layout_of(tokens, vocab, cols).bytes; }

cudaError_t launch_embedding_grad(const EmbedGradArgs &a, cudaStream_t stream)
{
    const GradLayout l = layout_of(a.tokens, a.vocab, a.cols);
    uint8_t *base = static_cast<uint8_t *>(a.work);
    GradArgs g{a, 8, 0, 0, 0, 1, l.slices, 0, l.pieces, a.tokens <= kFew, base + l.list,
               reinterpret_cast<Place *>(base + l.order), reinterpret_cast<int2 *>(base + l.rows), reinterpret_cast<int *>(base + l.counts), reinterpret_cast<int *>(base + l.valid),
               reinterpret_cast<float *>(base + l.partial)};
    // Neighbouring rows that are short together go to one CTA, as long as there are blocks for all CTAs.
    while ((a.cols << g.fold) < 256 && (a.vocab >> (g.fold + g.shift)) >= 2) ++g.fold;
    while (((((a.vocab + (1 << g.fold) - 1) >> g.fold) + (int64_t(1) << g.shift) - 1) >> g.shift << g.fold) > kOwnRows) ++g.shift;
    const int64_t ctas = std::min<int64_t>(int64_t(1) << g.shift, (a.vocab + (int64_t(1) << g.fold) - 1) >> g.fold);
    static std::atomic<uint64_t> asked[2] = {};
    const auto kernel = a.tokens > kBits ? novak_embedding_order_kernel<true> : novak_embedding_order_kernel<false>;
    cudaError_t e = ask_shared_memory(kernel, sizeof(OwnShared), asked[a.tokens > kBits]);
    if (e == cudaSuccess && !g.few)
        e = launch(kernel, dim3(static_cast<unsigned>((ctas + kCluster - 1) / kCluster * kCluster)), kOwnThreads, sizeof(OwnShared), stream, g);
    if (e != cudaSuccess) return e;

    const bool aligned = (a.tokens == 0 || wide(a.dout, a.type, a.tokens)) && wide(a.dtable, a.grad_type, a.vocab) && a.cols % 8 == 0;
    g.lanes = power((a.cols + 7) / 8, 32);
    const int lanes = aligned ? g.lanes : 32;
    g.steps = (a.cols + 8 * lanes - 1) / (8 * lanes);
    // as many rows as leave two rounds of warps (148 SMs with 32 each) something to do
    g.each = 1;
    while (g.each < std::min(kMostRows, lanes) && a.vocab * g.steps / (2 * g.each * (32 / lanes)) >= 148 * 32 * 2) g.each *= 2;
    g.group = std::max(power((std::min<int64_t>(a.cols, kSlice) + 7) / 8, kSlice / 8), 32);
    const int which = a.type * 4 + a.grad_type * 2 + aligned;
    return which == 0   ? launch_grad<0, 0, false>(g, stream)
           : which == 1 ? launch_grad<0, 0, true>(g, stream)
           : which == 2 ? launch_grad<0, 1, false>(g, stream)
           : which == 3 ? launch_grad<0, 1, true>(g, stream)
           : which == 4 ? launch_grad<1, 0, false>(g, stream)
           : which == 5 ? launch_grad<1, 0, true>(g, stream)
           : which == 6 ? launch_grad<1, 1, false>(g, stream)
                        : launch_grad<1, 1, true>(g, stream);
}

}  // namespace novak
