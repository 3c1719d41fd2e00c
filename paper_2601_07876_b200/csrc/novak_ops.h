// Internal interface between the host side of the training operators
// (novak_ops_host.cpp: checks, error text) and their kernels.  Not part
// of the C ABI.  A launcher is only called with rows >= 1 unless it says so, and
// with arguments that the host side has checked.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

namespace novak {

constexpr int kActBlock = 32;     // elements that share an exponent byte

inline int64_t act_pitch(int64_t cols) { return (cols + kActBlock - 1) / kActBlock * kActBlock; }

struct Mat {            // a caller's matrix; ptr may be NULL
    void *ptr;
    int64_t stride;     // elements between rows
};

struct Codes {          // an 8-bit form; both NULL or both set
    int8_t *codes;
    uint8_t *exps;
};

// Whether a matrix can be read 16 bytes at a time, 8 elements per thread.
inline bool wide(const Mat &m, int type, int64_t rows)
{
    const int64_t size = type == 0 ? 4 : 2;
    return (reinterpret_cast<uintptr_t>(m.ptr) & 15u) == 0 && (rows <= 1 || m.stride * size % 16 == 0);
}

// novak_act8.cu.  kind < 0: no function (packing); a, u_codes, a_codes may be NULL.
cudaError_t launch_activation(Mat u, Mat a, int type, int kind, Codes u_codes, Codes a_codes, int64_t rows,
                              int64_t cols, cudaStream_t stream);
// kind < 0: unpacking (da NULL); otherwise u or codes is NULL.
cudaError_t launch_activation_backward(Mat da, Mat u, int type, int kind, Codes codes, Mat du, int64_t rows,
                                       int64_t cols, cudaStream_t stream);

// novak_layer_norm.cu
struct NormArgs {
    Mat x, y;
    int type;
    const void *weight, *bias;
    int param_type;
    float eps;
    float *mean, *rstd;
    Codes codes;
    int64_t rows, cols;
};
cudaError_t launch_layer_norm(const NormArgs &a, cudaStream_t stream);

struct NormBackArgs {
    Mat dy, x;
    int type;
    const float *mean, *rstd;
    Codes codes;
    const void *weight;
    int param_type;
    Mat dx;
    void *dweight, *dbias;
    int grad_type;
    float *work;
    int64_t rows, cols;     // rows may be 0
};
size_t layer_norm_backward_bytes(int64_t rows, int64_t cols);
cudaError_t launch_layer_norm_backward(const NormBackArgs &a, cudaStream_t stream);

// novak_rms_norm.cu
struct RmsArgs {
    Mat x, residual, h, y;      // residual and h: both or neither
    int type;
    const void *weight;
    int param_type;
    float eps;
    float *rstd;
    Codes codes;
    int64_t rows, cols;
};
cudaError_t launch_rms_norm(const RmsArgs &a, cudaStream_t stream);

struct RmsBackArgs {
    Mat dy, dh, h;              // dh may be NULL; h or codes
    int type;
    const float *rstd;
    Codes codes;
    const void *weight;
    int param_type;
    Mat dx;
    void *dweight;
    int grad_type;
    float *work;
    int64_t rows, cols;         // rows may be 0
};
size_t rms_norm_backward_bytes(int64_t rows, int64_t cols);
cudaError_t launch_rms_norm_backward(const RmsBackArgs &a, cudaStream_t stream);

// novak_embedding.cu
struct EmbedArgs {
    const void *ids;
    int id_type;
    Mat table;
    int table_type;
    float scale;
    Mat out;
    int out_type;
    int64_t tokens, vocab, cols;
};
cudaError_t launch_embedding(const EmbedArgs &a, cudaStream_t stream);

struct EmbedGradArgs {
    Mat dout;
    int type;
    const void *ids;
    int id_type;
    float scale;
    Mat dtable;
    int grad_type, add;
    void *work;
    int64_t tokens, vocab, cols;    // tokens may be 0
};
size_t embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t cols);
cudaError_t launch_embedding_grad(const EmbedGradArgs &a, cudaStream_t stream);

// novak_orthogonalize.cu
constexpr int kMostSteps = 32;
struct OrthArgs {               // arrays of n on the host
    const void *const *g;
    const int64_t *g_stride;    // NULL: dense
    int type;
    void *const *out;           // bf16; or NULL, and theta is stepped
    const int64_t *out_stride;
    const int64_t *rows, *cols;
    int n;
    float coefficients[kMostSteps][3];
    int steps;
    double eps;
    float *const *theta, *const *m;
    float momentum;
    bool nesterov;
    const double *step;
    float decay;
    void *work;
    bool fine = false;          // operands of two parts in the large ones' products too
    int64_t withheld = -1;      // a tile whose end is not announced (a test of the waits' limit)
    uint64_t wait_ns = 0;       // a wait's limit; 0: the usual one
};
// 0: the matrices are too large or too many to be addressed.  `all`: where a.withheld >= 0, with which small matrices
// need a place too.
size_t orthogonalize_bytes(const int64_t *rows, const int64_t *cols, int n, bool fine, bool all = false);
cudaError_t orthogonalize_gave_up(unsigned *count, cudaStream_t stream);
cudaError_t launch_orthogonalize(const OrthArgs &a, cudaStream_t stream);

// novak_weight_grad.cu
struct WeightGradArgs {
    Mat dy;
    int type;
    Codes codes;
    const void *weight, *bias;
    int param_type;
    void *dw, *db;
    int grad_type;
    void *work;
    int64_t rows, n_out, n_in;     // rows may be 0
    uint64_t wait_ns = 0;          // a wait's limit; 0: the usual one
    int withheld = -1;             // pair of SMs whose first sum is not announced (a test of the limit)
};
// Pairs of SMs that work on it; 0: the ordinary cores do, and wait for nothing.
int weight_grad_pairs(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in);
size_t weight_grad_bytes(const Mat &dy, int type, int64_t rows, int64_t n_out, int64_t n_in);
cudaError_t weight_grad_gave_up(unsigned *count, cudaStream_t stream);
cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t stream);

}  // namespace novak
