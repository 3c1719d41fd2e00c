// Token embedding, out[t] = scale table[ids[t]], and its gradient, the sum of dout's rows
// over the tokens of an id.
#include <algorithm>

#include "novak_ops.cuh"

namespace novak {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t id_at(const void *ids, int type, int64_t t)
{
    return type == NOVAK_ID_I32 ? static_cast<const int32_t *>(ids)[t] : static_cast<const int64_t *>(ids)[t];
}

// A warp per token.
template <int TABLE, int OUT, bool WIDE>
__global__ void __launch_bounds__(kThreads) novak_embedding_kernel(EmbedArgs a)
{
    using T = typename Elem<TABLE>::T;
    using O = typename Elem<OUT>::T;
    start();
    const int lane = threadIdx.x % 32;
    for (int64_t t = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / 32; t < a.tokens;
         t += static_cast<int64_t>(gridDim.x) * (kThreads / 32)) {
        const int64_t id = id_at(a.ids, a.id_type, t);
        const bool there = id >= 0 && id < a.vocab;
        const T *row = static_cast<const T *>(a.table.ptr) + (there ? id : 0) * a.table.stride;
        for (int64_t c = lane * 8; c < a.cols; c += 256) {
            float v[8] = {};
            if (there) load8<WIDE>(row, c, a.cols, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= there ? a.scale : 0.0f;
            store8<WIDE>(static_cast<O *>(a.out.ptr) + t * a.out.stride, c, a.cols, v);
        }
    }
}

// A CTA per row of the table looks through all ids.
template <int TYPE> __global__ void __launch_bounds__(kThreads) novak_embedding_grad_kernel(EmbedGradArgs a)
{
    using T = typename Elem<TYPE>::T;
    __shared__ int found[kThreads / 32];
    start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x)
        for (int64_t c0 = 0; c0 < a.cols; c0 += kThreads) {
            const int64_t c = c0 + threadIdx.x;
            float sum = 0.0f;
            bool any = false;
            for (int64_t t0 = 0; t0 < a.tokens; t0 += kThreads) {
                const int64_t t = t0 + threadIdx.x;
                const unsigned hit = __ballot_sync(0xffffffffu, t < a.tokens && id_at(a.ids, a.id_type, t) == v);
                __syncthreads();
                if (lane == 0) found[warp] = static_cast<int>(hit);
                __syncthreads();
                for (int w = 0; w < kThreads / 32; ++w)
                    for (unsigned m = static_cast<unsigned>(found[w]); m; m &= m - 1) {
                        const int64_t at = t0 + w * 32 + __ffs(static_cast<int>(m)) - 1;
                        any = true;
                        if (c < a.cols) sum += to_float(static_cast<const T *>(a.dout.ptr)[at * a.dout.stride + c]);
                    }
            }
            if (c >= a.cols || (a.add && !any)) continue;
            const int64_t at = v * a.dtable.stride + c;
            store_param(a.dtable.ptr, a.grad_type, at, a.add ? fmaf(sum, a.scale, param_at(a.dtable.ptr, a.grad_type, at)) : sum * a.scale);
        }
}

}  // namespace

cudaError_t launch_embedding(const EmbedArgs &a, cudaStream_t stream)
{
    const bool w = wide(a.table, a.table_type, a.vocab) && wide(a.out, a.out_type, a.tokens);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.tokens + kThreads / 32 - 1) / (kThreads / 32), 148 * 8)));
    const int which = a.table_type * 4 + a.out_type * 2 + w;
    auto kernel = which == 0   ? novak_embedding_kernel<0, 0, false>
                  : which == 1 ? novak_embedding_kernel<0, 0, true>
                  : which == 2 ? novak_embedding_kernel<0, 1, false>
                  : which == 3 ? novak_embedding_kernel<0, 1, true>
                  : which == 4 ? novak_embedding_kernel<1, 0, false>
                  : which == 5 ? novak_embedding_kernel<1, 0, true>
                  : which == 6 ? novak_embedding_kernel<1, 1, false>
                               : novak_embedding_kernel<1, 1, true>;
    return launch(kernel, grid, kThreads, 0, stream, a);
}

size_t embedding_grad_bytes(int64_t, int64_t, int64_t) { return 0; }

cudaError_t launch_embedding_grad(const EmbedGradArgs &a, cudaStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.vocab, 148 * 8)));
    return launch(a.type == NOVAK_TYPE_F32 ? novak_embedding_grad_kernel<0> : novak_embedding_grad_kernel<1>, grid, kThreads, 0, stream, a);
}

}  // namespace novak
