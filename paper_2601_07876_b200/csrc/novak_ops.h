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
