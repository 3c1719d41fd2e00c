// Host side of the training operators' C entry points: argument checks and
// error text.  The launchers are in novak_act8.cu,
// novak_layer_norm.cu and novak_weight_grad.cu.
#include "novak.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "novak_ops.h"

using namespace novak;

namespace {

thread_local char g_ops_error[256] = "";

int refuse(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_ops_error, sizeof g_ops_error, fmt, ap);
    va_end(ap);
    return NOVAK_EINVAL;
}

int finish(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return NOVAK_OK;
    std::snprintf(g_ops_error, sizeof g_ops_error, "%s: %s", what, cudaGetErrorString(e));
    return NOVAK_ECUDA;
}

bool is_type(int t) { return t == NOVAK_TYPE_F32 || t == NOVAK_TYPE_BF16; }

constexpr int64_t kMaxDim = int64_t(1) << 40;    // products of two stay below 2^63 with kMaxElems
constexpr int64_t kMaxElems = int64_t(1) << 60;

int check_shape(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1) return refuse("rows must be >= 0 and the other sizes >= 1");
    if (rows > kMaxDim || cols > kMaxDim || (rows > 0 && act_pitch(cols) > kMaxElems / rows))
        return refuse("a matrix of %lld x %lld elements cannot be addressed", static_cast<long long>(rows),
                      static_cast<long long>(cols));
    return NOVAK_OK;
}

int check_mat(const char *name, const Mat &m, int type, int64_t rows, int64_t cols)
{
    if (rows == 0) return NOVAK_OK;
    if (!m.ptr) return refuse("%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(m.ptr) % (type == NOVAK_TYPE_F32 ? 4 : 2))
        return refuse("%s is not aligned to its elements", name);
    if (rows > 1 && (m.stride < cols || m.stride > kMaxElems / rows))
        return refuse("%s: stride %lld for rows of %lld elements", name, static_cast<long long>(m.stride),
                      static_cast<long long>(cols));
    return NOVAK_OK;
}

// `needed`: an absent form is an error.
int check_codes(const char *name, const Codes &c, int64_t rows, bool needed)
{
    if (rows == 0) return NOVAK_OK;
    if ((c.codes == nullptr) != (c.exps == nullptr)) return refuse("%s: codes and exps come together", name);
    if (!c.codes) return needed ? refuse("%s: codes is NULL", name) : NOVAK_OK;
    if (reinterpret_cast<uintptr_t>(c.codes) & 31u) return refuse("%s: codes are not 32-byte aligned", name);
    return NOVAK_OK;
}

int check_vector(const char *name, const void *p, int type)
{
    if (!is_type(type)) return refuse("bad type of %s", name);
    if (!p) return refuse("%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % (type == NOVAK_TYPE_F32 ? 4 : 2))
        return refuse("%s is not aligned to its elements", name);
    return NOVAK_OK;
}

int check_floats(const char *name, const float *p)
{
    return reinterpret_cast<uintptr_t>(p) & 3u ? refuse("%s is not 4-byte aligned", name) : int(NOVAK_OK);
}

Mat mat(const void *p, int64_t stride) { return Mat{const_cast<void *>(p), stride}; }
Codes form(const int8_t *c, const uint8_t *e) { return Codes{const_cast<int8_t *>(c), const_cast<uint8_t *>(e)}; }

#define CHECK(call)                         \
    do {                                    \
        const int check_rc = (call);        \
        if (check_rc != NOVAK_OK) return check_rc; \
    } while (0)

int check_weight_grad_sizes(int64_t rows, int64_t n_out, int64_t n_in)
{
    CHECK(check_shape(rows, n_out));
    CHECK(check_shape(rows, n_in));
    if (rows > INT32_MAX || n_out > (1 << 22) || n_in > (1 << 22))
        return refuse("sizes of up to 2^31 - 1 rows and 2^22 inputs and outputs are taken");
    return NOVAK_OK;
}

int check_weight_grad(const WeightGradArgs &a, size_t work_bytes)
{
    if (!is_type(a.type)) return refuse("bad type");
    CHECK(check_weight_grad_sizes(a.rows, a.n_out, a.n_in));
    CHECK(check_mat("dy", a.dy, a.type, a.rows, a.n_out));
    CHECK(check_codes("x", a.codes, a.rows, true));
    if ((a.weight != nullptr) != (a.bias != nullptr)) return refuse("the norm's weight and bias come together");
    if (a.weight) {
        CHECK(check_vector("weight", a.weight, a.param_type));
        CHECK(check_vector("bias", a.bias, a.param_type));
    }
    CHECK(check_vector("dw", a.dw, a.grad_type));
    if (a.db) CHECK(check_vector("db", a.db, a.grad_type));
    const size_t need = weight_grad_bytes(a.dy, a.type, a.rows, a.n_out, a.n_in);
    if (need > 0 && (!a.work || work_bytes < need || (reinterpret_cast<uintptr_t>(a.work) & 255u)))
        return refuse("work: %zu bytes, 256-byte aligned, are needed", need);
    return NOVAK_OK;
}

}  // namespace

extern "C" {

const char *novak_ops_error(void) { return g_ops_error; }

int novak_ops_gave_up(unsigned *count, void *stream)
{
    if (!count) return refuse("count is NULL");
    return finish(weight_grad_gave_up(count, static_cast<cudaStream_t>(stream)), "novak_ops_gave_up");
}

int64_t novak_act8_pitch(int64_t cols) { return cols < 1 || cols > kMaxDim ? 0 : act_pitch(cols); }

int novak_act8_pack(const void *d_x, int64_t x_stride, int type, int8_t *d_codes, uint8_t *d_exps,
                    int64_t rows, int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("x", mat(d_x, x_stride), type, rows, cols));
    CHECK(check_codes("x", form(d_codes, d_exps), rows, true));
    if (rows == 0) return NOVAK_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish(launch_activation(mat(d_x, x_stride), Mat{}, type, -1, form(d_codes, d_exps), Codes{}, rows,
                                    cols, s), "novak_act8_pack");
}

int novak_act8_unpack(const int8_t *d_codes, const uint8_t *d_exps, void *d_out, int64_t out_stride,
                      int type, int64_t rows, int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("out", mat(d_out, out_stride), type, rows, cols));
    CHECK(check_codes("out", form(d_codes, d_exps), rows, true));
    if (rows == 0) return NOVAK_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish(launch_activation_backward(Mat{}, Mat{}, type, -1, form(d_codes, d_exps),
                                             mat(d_out, out_stride), rows, cols, s), "novak_act8_unpack");
}

int novak_layer_norm(const void *d_x, int64_t x_stride, void *d_y, int64_t y_stride, int type,
                     const void *d_weight, const void *d_bias, int param_type, double eps,
                     float *d_mean, float *d_rstd, int8_t *d_codes, uint8_t *d_exps, int64_t rows,
                     int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    if (!(eps >= 0.0) || !std::isfinite(eps)) return refuse("eps must be >= 0 and finite");
    CHECK(check_mat("x", mat(d_x, x_stride), type, rows, cols));
    CHECK(check_mat("y", mat(d_y, y_stride), type, rows, cols));
    CHECK(check_vector("weight", d_weight, param_type));
    if (d_bias) CHECK(check_vector("bias", d_bias, param_type));
    CHECK(check_floats("mean", d_mean));
    CHECK(check_floats("rstd", d_rstd));
    CHECK(check_codes("xhat", form(d_codes, d_exps), rows, false));
    if (rows == 0) return NOVAK_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormArgs a{mat(d_x, x_stride), mat(d_y, y_stride), type, d_weight, d_bias, param_type,
                     static_cast<float>(eps), d_mean, d_rstd, form(d_codes, d_exps), rows, cols};
    return finish(launch_layer_norm(a, s), "novak_layer_norm");
}

size_t novak_layer_norm_backward_bytes(int64_t rows, int64_t cols)
{
    return check_shape(rows, cols) == NOVAK_OK ? layer_norm_backward_bytes(rows, cols) : 0;
}

int novak_layer_norm_backward(const void *d_dy, int64_t dy_stride, const void *d_x, int64_t x_stride,
                              int type, const float *d_mean, const float *d_rstd,
                              const int8_t *d_codes, const uint8_t *d_exps, const void *d_weight,
                              int param_type, void *d_dx, int64_t dx_stride, void *d_dweight,
                              void *d_dbias, int grad_type, void *d_work, size_t work_bytes,
                              int64_t rows, int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("dy", mat(d_dy, dy_stride), type, rows, cols));
    CHECK(check_mat("dx", mat(d_dx, dx_stride), type, rows, cols));
    CHECK(check_vector("weight", d_weight, param_type));
    if (d_dweight) CHECK(check_vector("dweight", d_dweight, grad_type));
    if (d_dbias) CHECK(check_vector("dbias", d_dbias, grad_type));
    CHECK(check_codes("xhat", form(d_codes, d_exps), rows, false));
    if (rows > 0) {
        if ((d_codes != nullptr) == (d_x != nullptr)) return refuse("xhat comes from its 8-bit form or from x: one of the two");
        if ((d_x != nullptr) != (d_mean != nullptr)) return refuse("x and mean come together");
        if (d_x) CHECK(check_mat("x", mat(d_x, x_stride), type, rows, cols));
        if (!d_rstd) return refuse("rstd is NULL");
    }
    CHECK(check_floats("mean", d_mean));
    CHECK(check_floats("rstd", d_rstd));
    const size_t need = layer_norm_backward_bytes(rows, cols);
    if (need > 0 && (!d_work || work_bytes < need || (reinterpret_cast<uintptr_t>(d_work) & 15u)))
        return refuse("work: %zu bytes, 16-byte aligned, are needed", need);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormBackArgs a{mat(d_dy, dy_stride), mat(d_x, x_stride), type, d_mean, d_rstd, form(d_codes, d_exps),
                         d_weight, param_type, mat(d_dx, dx_stride), d_dweight, d_dbias, grad_type,
                         static_cast<float *>(d_work), rows, cols};
    return finish(launch_layer_norm_backward(a, s), "novak_layer_norm_backward");
}

int novak_activation(const void *d_u, int64_t u_stride, void *d_a, int64_t a_stride, int type, int kind,
                     int8_t *d_u_codes, uint8_t *d_u_exps, int8_t *d_a_codes, uint8_t *d_a_exps,
                     int64_t rows, int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    if (kind < NOVAK_ACT_GELU || kind > NOVAK_ACT_SILU) return refuse("no activation function %d", kind);
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("u", mat(d_u, u_stride), type, rows, cols));
    if (d_a) CHECK(check_mat("a", mat(d_a, a_stride), type, rows, cols));
    CHECK(check_codes("u", form(d_u_codes, d_u_exps), rows, false));
    CHECK(check_codes("a", form(d_a_codes, d_a_exps), rows, false));
    if (rows == 0 || (!d_a && !d_u_codes && !d_a_codes)) return NOVAK_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish(launch_activation(mat(d_u, u_stride), mat(d_a, a_stride), type, kind, form(d_u_codes, d_u_exps),
                                    form(d_a_codes, d_a_exps), rows, cols, s), "novak_activation");
}

int novak_activation_backward(const void *d_da, int64_t da_stride, const void *d_u, int64_t u_stride,
                              int type, int kind, const int8_t *d_codes, const uint8_t *d_exps,
                              void *d_du, int64_t du_stride, int64_t rows, int64_t cols, void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    if (kind < NOVAK_ACT_GELU || kind > NOVAK_ACT_SILU) return refuse("no activation function %d", kind);
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("da", mat(d_da, da_stride), type, rows, cols));
    CHECK(check_mat("du", mat(d_du, du_stride), type, rows, cols));
    CHECK(check_codes("u", form(d_codes, d_exps), rows, false));
    if (rows == 0) return NOVAK_OK;
    if ((d_codes != nullptr) == (d_u != nullptr)) return refuse("u comes from its 8-bit form or as it is: one of the two");
    if (d_u) CHECK(check_mat("u", mat(d_u, u_stride), type, rows, cols));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish(launch_activation_backward(mat(d_da, da_stride), mat(d_u, u_stride), type, kind,
                                             form(d_codes, d_exps), mat(d_du, du_stride), rows, cols, s),
                  "novak_activation_backward");
}

size_t novak_linear_weight_grad_bytes(const void *d_dy, int64_t dy_stride, int type, int64_t rows,
                                      int64_t n_out, int64_t n_in)
{
    if (!is_type(type) || check_weight_grad_sizes(rows, n_out, n_in) != NOVAK_OK) return 0;
    return weight_grad_bytes(mat(d_dy, dy_stride), type, rows, n_out, n_in);
}

int novak_linear_weight_grad(const void *d_dy, int64_t dy_stride, int type, const int8_t *d_codes,
                             const uint8_t *d_exps, const void *d_weight, const void *d_bias,
                             int param_type, void *d_dw, void *d_db, int grad_type, void *d_work,
                             size_t work_bytes, int64_t rows, int64_t n_out, int64_t n_in,
                             void *stream)
{
    const WeightGradArgs a{mat(d_dy, dy_stride), type, form(d_codes, d_exps), d_weight, d_bias, param_type, d_dw, d_db,
                           grad_type, d_work, rows, n_out, n_in};
    CHECK(check_weight_grad(a, work_bytes));
    return finish(launch_weight_grad(a, static_cast<cudaStream_t>(stream)), "novak_linear_weight_grad");
}

int novak_selftest_weight_grad_wait(const void *d_dy, int64_t dy_stride, int type, const int8_t *d_codes,
                                    const uint8_t *d_exps, const void *d_weight, const void *d_bias,
                                    int param_type, void *d_dw, void *d_db, int grad_type, void *d_work,
                                    size_t work_bytes, int64_t rows, int64_t n_out, int64_t n_in, int pair,
                                    uint64_t wait_ns, void *stream)
{
    const WeightGradArgs a{mat(d_dy, dy_stride), type, form(d_codes, d_exps), d_weight, d_bias, param_type, d_dw, d_db,
                           grad_type, d_work, rows, n_out, n_in, wait_ns, pair};
    CHECK(check_weight_grad(a, work_bytes));
    const int pairs = weight_grad_pairs(a.dy, type, rows, n_out, n_in);
    if (pair < 0 || pair >= pairs) return refuse("pair %d of %d", pair, pairs);
    return finish(launch_weight_grad(a, static_cast<cudaStream_t>(stream)), "novak_selftest_weight_grad_wait");
}

}  // extern "C"
