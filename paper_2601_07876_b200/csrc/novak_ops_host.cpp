// Host side of the training operators' C entry points: argument checks and
// error text.  The launchers are in novak_act8.cu, novak_layer_norm.cu,
// novak_rms_norm.cu, novak_embedding.cu, novak_orthogonalize.cu and novak_weight_grad.cu.
#include "novak.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <memory>
#include <new>
#include <utility>

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

bool is_id(int t) { return t == NOVAK_ID_I32 || t == NOVAK_ID_I64; }

int check_ids(const void *ids, int id_type, int64_t tokens)
{
    if (!is_id(id_type)) return refuse("bad type of ids");
    if (tokens == 0) return NOVAK_OK;
    if (!ids) return refuse("ids is NULL");
    if (reinterpret_cast<uintptr_t>(ids) % (id_type == NOVAK_ID_I32 ? 4 : 8)) return refuse("ids are not aligned to their elements");
    return NOVAK_OK;
}

int check_embedding_sizes(int64_t tokens, int64_t vocab, int64_t cols)
{
    CHECK(check_shape(tokens, cols));
    CHECK(check_shape(vocab, cols));
    if (tokens > INT32_MAX || vocab > INT32_MAX || cols > INT32_MAX) return refuse("up to 2^31 - 1 tokens, rows of the table and columns are taken");
    return NOVAK_OK;
}

int check_scale(double scale)
{
    return std::isfinite(static_cast<float>(scale)) ? int(NOVAK_OK) : refuse("scale must be finite (in fp32)");
}

// How large |x (a + b x^2 + c x^4)| and |b t + c t^2|, t = x^2, get on [0, r]: at the ends, or
// where the derivatives a + 3 b t + 5 c t^2 and b + 2 c t are zero.  (Roots from the sum that does not cancel, so that they
// hold for any ratio of the coefficients, and of coefficients scaled to 1, so that no square overflows.)
void reach(const double *abc, double r, double &value, double &product)
{
    const double a = abc[0], b = abc[1], c = abc[2], top = r * r;
    const auto at = [&](double t) {
        if (!(t > 0.0 && t <= top)) return;
        value = std::max(value, std::fabs(std::sqrt(t) * (a + t * (b + t * c))));
        product = std::max(product, std::fabs(t * (b + t * c)));
    };
    value = product = 0.0;
    at(top);
    if (c != 0.0) at(-b / (2.0 * c));
    const double most = std::max({std::fabs(a), std::fabs(b), std::fabs(c)});
    if (most == 0.0) return;
    const double a1 = a / most, b1 = b / most, c1 = c / most, d = 9.0 * b1 * b1 - 20.0 * a1 * c1;
    if (d < 0.0) return;
    const double q = -(3.0 * b1 + std::copysign(std::sqrt(d), b1)) / 2.0;
    if (c1 != 0.0) at(q / (5.0 * c1));
    if (q != 0.0) at(a1 / q);
}

// Everything about the matrices but where they lie.
int check_orthogonalize(const int64_t *rows, const int64_t *cols, int n, const double *coefficients, int steps, double eps)
{
    if (n < 0 || n > (1 << 14)) return refuse("0 to 2^14 matrices are taken");
    if (n > 0 && (!rows || !cols)) return refuse("rows or cols is NULL");
    for (int i = 0; i < n; ++i)
        if (rows[i] < 0 || cols[i] < 0 || rows[i] > (1 << 16) || cols[i] > (1 << 16))
            return refuse("matrix %d: up to 2^16 rows and columns are taken", i);
    if (steps < 1 || steps > kMostSteps) return refuse("1 to %d steps are taken", kMostSteps);
    if (!coefficients) return refuse("coefficients is NULL");
    if (!(eps >= 0.0) || !std::isfinite(eps)) return refuse("eps must be >= 0 and finite");
    double r = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double *abc = coefficients + 3 * k;
        if (!std::isfinite(abc[0]) || !std::isfinite(abc[1]) || !std::isfinite(abc[2])) return refuse("coefficients must be finite");
        double product;
        reach(abc, 1.01 * r, r, product);       // (1 %: what the products are rounded by)
        if (!(r <= 4.0 && product <= 15.0))
            return refuse("step %d: singular values of up to %.3g, and up to %.3g of b A + c A^2 (4 and 15 are held)", k, r, product);
    }
    return NOVAK_OK;
}

int check_orthogonalize_work(const OrthArgs &a, size_t work_bytes)
{
    const size_t need = orthogonalize_bytes(a.rows, a.cols, a.n, a.fine);
    bool any = false;
    for (int i = 0; i < a.n; ++i) any |= a.rows[i] > 0 && a.cols[i] > 0;
    if (any && need == 0) return refuse("the matrices are more than can be addressed in one call");
    if (need > 0 && (!a.work || work_bytes < need || (reinterpret_cast<uintptr_t>(a.work) & 255u)))
        return refuse("work: %zu bytes, 256-byte aligned, are needed", need);
    return NOVAK_OK;
}

void set_coefficients(OrthArgs &a, const double *coefficients, int steps)
{
    a.steps = steps;
    for (int k = 0; k < 3 * steps; ++k) a.coefficients[k / 3][k % 3] = static_cast<float>(coefficients[k]);
}

int orthogonalize(OrthArgs &a, const double *coefficients, int steps, size_t work_bytes, void *stream, const char *where)
{
    if (!is_type(a.type)) return refuse("bad type");
    CHECK(check_orthogonalize(a.rows, a.cols, a.n, coefficients, steps, a.eps));
    if (a.n > 0 && (!a.g || !a.g_stride || !a.out || !a.out_stride)) return refuse("an array is NULL");
    for (int i = 0; i < a.n; ++i) {
        if (a.cols[i] == 0) continue;
        CHECK(check_mat("g", mat(a.g[i], a.g_stride[i]), a.type, a.rows[i], a.cols[i]));
        CHECK(check_mat("out", mat(a.out[i], a.out_stride[i]), NOVAK_TYPE_BF16, a.rows[i], a.cols[i]));
    }
    set_coefficients(a, coefficients, steps);
    CHECK(check_orthogonalize_work(a, work_bytes));
    return finish(launch_orthogonalize(a, static_cast<cudaStream_t>(stream)), where);
}

size_t workspace(const int64_t *rows, const int64_t *cols, int n, bool fine)
{
    const double one[3] = {1.0, 0.0, 0.0};
    return check_orthogonalize(rows, cols, n, one, 1, 0.0) == NOVAK_OK ? orthogonalize_bytes(rows, cols, n, fine) : 0;
}

int orthogonal_step(float *const *d_theta, const void *const *d_g, int grad_type, float *const *d_m, const int64_t *rows,
                    const int64_t *cols, int n, double momentum, int nesterov, const double *step, double decay,
                    const double *coefficients, int steps, double eps, void *d_work, size_t work_bytes, bool fine, void *stream,
                    const char *where)
{
    if (!is_type(grad_type)) return refuse("bad type");
    CHECK(check_orthogonalize(rows, cols, n, coefficients, steps, eps));
    if (!(momentum >= 0.0 && momentum < 1.0)) return refuse("momentum must be in [0, 1)");
    if (!std::isfinite(decay)) return refuse("decay must be finite");
    if (n > 0 && (!d_theta || !d_g || !d_m || !step)) return refuse("an array is NULL");
    for (int i = 0; i < n; ++i) {
        if (!std::isfinite(step[i])) return refuse("step must be finite");
        if (cols[i] == 0) continue;
        CHECK(check_mat("theta", mat(d_theta[i], cols[i]), NOVAK_TYPE_F32, rows[i], cols[i]));
        CHECK(check_mat("m", mat(d_m[i], cols[i]), NOVAK_TYPE_F32, rows[i], cols[i]));
        CHECK(check_mat("g", mat(d_g[i], cols[i]), grad_type, rows[i], cols[i]));
    }
    // what is written belongs to one matrix alone
    using Range = std::pair<uintptr_t, uintptr_t>;
    const std::unique_ptr<Range[]> written(new (std::nothrow) Range[2 * static_cast<size_t>(n) + 1]);
    if (!written) return refuse("no memory on the host");
    Range *end = written.get();
    const auto range = [&](const void *p, int i, size_t size) {
        const uintptr_t first = reinterpret_cast<uintptr_t>(p);
        return Range(first, first + static_cast<size_t>(rows[i]) * static_cast<size_t>(cols[i]) * size);
    };
    for (int i = 0; i < n; ++i)
        if (rows[i] > 0 && cols[i] > 0)
            for (const float *p : {d_theta[i], d_m[i]}) *end++ = range(p, i, sizeof(float));
    std::sort(written.get(), end);
    for (const Range *r = written.get() + 1; r < end; ++r)
        if (r->first < r[-1].second) return refuse("theta and m overlap one another");
    for (int i = 0; i < n; ++i) {
        if (rows[i] == 0 || cols[i] == 0) continue;
        const Range g = range(d_g[i], i, grad_type == NOVAK_TYPE_F32 ? 4 : 2);
        const Range *behind = std::lower_bound(written.get(), end, Range(g.second, 0));     // the first that begins behind g
        if (behind != written.get() && behind[-1].second > g.first) return refuse("g overlaps theta or m");
    }
    OrthArgs a{d_g, nullptr, grad_type, nullptr, nullptr, rows, cols, n, {}, 0, eps, d_theta, d_m,
               static_cast<float>(momentum), nesterov != 0, step, static_cast<float>(decay), d_work, fine};
    set_coefficients(a, coefficients, steps);
    CHECK(check_orthogonalize_work(a, work_bytes));
    return finish(launch_orthogonalize(a, static_cast<cudaStream_t>(stream)), where);
}

}  // namespace

extern "C" {

const char *novak_ops_error(void) { return g_ops_error; }

int novak_ops_gave_up(unsigned *count, void *stream)
{
    if (!count) return refuse("count is NULL");
    unsigned more = 0;
    cudaError_t e = weight_grad_gave_up(count, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) e = orthogonalize_gave_up(&more, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) *count += more;
    return finish(e, "novak_ops_gave_up");
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

int novak_rms_norm(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, void *d_h,
                   int64_t h_stride, void *d_y, int64_t y_stride, int type, const void *d_weight, int param_type,
                   double eps, float *d_rstd, int8_t *d_codes, uint8_t *d_exps, int64_t rows, int64_t cols,
                   void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    if (!(eps >= 0.0) || !std::isfinite(eps)) return refuse("eps must be >= 0 and finite");
    CHECK(check_mat("x", mat(d_x, x_stride), type, rows, cols));
    CHECK(check_mat("y", mat(d_y, y_stride), type, rows, cols));
    if (rows > 0 && (d_residual != nullptr) != (d_h != nullptr)) return refuse("residual and h come together");
    if (d_residual) {
        CHECK(check_mat("residual", mat(d_residual, residual_stride), type, rows, cols));
        CHECK(check_mat("h", mat(d_h, h_stride), type, rows, cols));
        if (rows > 0 && d_h == d_y) return refuse("h and y are one");
    }
    CHECK(check_vector("weight", d_weight, param_type));
    CHECK(check_floats("rstd", d_rstd));
    CHECK(check_codes("xhat", form(d_codes, d_exps), rows, false));
    if (rows == 0) return NOVAK_OK;
    const RmsArgs a{mat(d_x, x_stride), mat(d_residual, residual_stride), mat(d_h, h_stride), mat(d_y, y_stride), type,
                    d_weight, param_type, static_cast<float>(eps), d_rstd, form(d_codes, d_exps), rows, cols};
    return finish(launch_rms_norm(a, static_cast<cudaStream_t>(stream)), "novak_rms_norm");
}

size_t novak_rms_norm_backward_bytes(int64_t rows, int64_t cols)
{
    return check_shape(rows, cols) == NOVAK_OK ? rms_norm_backward_bytes(rows, cols) : 0;
}

int novak_rms_norm_backward(const void *d_dy, int64_t dy_stride, const void *d_dh, int64_t dh_stride, const void *d_h,
                            int64_t h_stride, int type, const float *d_rstd, const int8_t *d_codes,
                            const uint8_t *d_exps, const void *d_weight, int param_type, void *d_dx, int64_t dx_stride,
                            void *d_dweight, int grad_type, void *d_work, size_t work_bytes, int64_t rows, int64_t cols,
                            void *stream)
{
    if (!is_type(type)) return refuse("bad type");
    CHECK(check_shape(rows, cols));
    CHECK(check_mat("dy", mat(d_dy, dy_stride), type, rows, cols));
    if (d_dh) CHECK(check_mat("dh", mat(d_dh, dh_stride), type, rows, cols));
    CHECK(check_mat("dx", mat(d_dx, dx_stride), type, rows, cols));
    CHECK(check_vector("weight", d_weight, param_type));
    if (d_dweight) CHECK(check_vector("dweight", d_dweight, grad_type));
    CHECK(check_codes("xhat", form(d_codes, d_exps), rows, false));
    if (rows > 0) {
        if ((d_codes != nullptr) == (d_h != nullptr)) return refuse("xhat comes from its 8-bit form or from h: one of the two");
        if (d_h) CHECK(check_mat("h", mat(d_h, h_stride), type, rows, cols));
        if (!d_rstd) return refuse("rstd is NULL");
    }
    CHECK(check_floats("rstd", d_rstd));
    const size_t need = rms_norm_backward_bytes(rows, cols);
    if (need > 0 && (!d_work || work_bytes < need || (reinterpret_cast<uintptr_t>(d_work) & 15u)))
        return refuse("work: %zu bytes, 16-byte aligned, are needed", need);
    const RmsBackArgs a{mat(d_dy, dy_stride), mat(d_dh, dh_stride), mat(d_h, h_stride), type, d_rstd, form(d_codes, d_exps),
                        d_weight, param_type, mat(d_dx, dx_stride), d_dweight, grad_type, static_cast<float *>(d_work),
                        rows, cols};
    return finish(launch_rms_norm_backward(a, static_cast<cudaStream_t>(stream)), "novak_rms_norm_backward");
}

int novak_embedding(const void *d_ids, int id_type, const void *d_table, int64_t table_stride, int table_type,
                    double scale, void *d_out, int64_t out_stride, int out_type, int64_t tokens, int64_t vocab,
                    int64_t cols, void *stream)
{
    if (!is_type(table_type) || !is_type(out_type)) return refuse("bad type");
    CHECK(check_embedding_sizes(tokens, vocab, cols));
    CHECK(check_ids(d_ids, id_type, tokens));
    if (tokens > 0) CHECK(check_mat("table", mat(d_table, table_stride), table_type, vocab, cols));
    CHECK(check_mat("out", mat(d_out, out_stride), out_type, tokens, cols));
    CHECK(check_scale(scale));
    if (tokens == 0) return NOVAK_OK;
    const EmbedArgs a{d_ids, id_type, mat(d_table, table_stride), table_type, static_cast<float>(scale),
                      mat(d_out, out_stride), out_type, tokens, vocab, cols};
    return finish(launch_embedding(a, static_cast<cudaStream_t>(stream)), "novak_embedding");
}

size_t novak_embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t cols)
{
    return check_embedding_sizes(tokens, vocab, cols) == NOVAK_OK ? embedding_grad_bytes(tokens, vocab, cols) : 0;
}

int novak_embedding_grad(const void *d_dout, int64_t dout_stride, int type, const void *d_ids, int id_type, double scale,
                         void *d_dtable, int64_t dtable_stride, int grad_type, int add, void *d_work, size_t work_bytes,
                         int64_t tokens, int64_t vocab, int64_t cols, void *stream)
{
    if (!is_type(type) || !is_type(grad_type)) return refuse("bad type");
    CHECK(check_embedding_sizes(tokens, vocab, cols));
    CHECK(check_ids(d_ids, id_type, tokens));
    CHECK(check_mat("dout", mat(d_dout, dout_stride), type, tokens, cols));
    CHECK(check_mat("dtable", mat(d_dtable, dtable_stride), grad_type, vocab, cols));
    CHECK(check_scale(scale));
    const size_t need = embedding_grad_bytes(tokens, vocab, cols);
    if (need > 0 && (!d_work || work_bytes < need || (reinterpret_cast<uintptr_t>(d_work) & 255u)))
        return refuse("work: %zu bytes, 256-byte aligned, are needed", need);
    if (vocab == 0 || (add && tokens == 0)) return NOVAK_OK;
    const EmbedGradArgs a{mat(d_dout, dout_stride), type, d_ids, id_type, static_cast<float>(scale),
                          mat(d_dtable, dtable_stride), grad_type, add != 0, d_work, tokens, vocab, cols};
    return finish(launch_embedding_grad(a, static_cast<cudaStream_t>(stream)), "novak_embedding_grad");
}

size_t novak_orthogonalize_bytes(const int64_t *rows, const int64_t *cols, int n) { return workspace(rows, cols, n, false); }

size_t novak_orthogonalize_fine_bytes(const int64_t *rows, const int64_t *cols, int n) { return workspace(rows, cols, n, true); }

int novak_orthogonalize(const void *const *d_g, const int64_t *g_stride, int type, void *const *d_out,
                        const int64_t *out_stride, const int64_t *rows, const int64_t *cols, int n,
                        const double *coefficients, int steps, double eps, void *d_work, size_t work_bytes, void *stream)
{
    OrthArgs a{d_g, g_stride, type, d_out, out_stride, rows, cols, n, {}, 0, eps, nullptr, nullptr, 0.0f, false, nullptr,
               0.0f, d_work};
    return orthogonalize(a, coefficients, steps, work_bytes, stream, "novak_orthogonalize");
}

int novak_orthogonalize_fine(const void *const *d_g, const int64_t *g_stride, int type, void *const *d_out,
                             const int64_t *out_stride, const int64_t *rows, const int64_t *cols, int n,
                             const double *coefficients, int steps, double eps, void *d_work, size_t work_bytes, void *stream)
{
    OrthArgs a{d_g, g_stride, type, d_out, out_stride, rows, cols, n, {}, 0, eps, nullptr, nullptr, 0.0f, false, nullptr,
               0.0f, d_work, true};
    return orthogonalize(a, coefficients, steps, work_bytes, stream, "novak_orthogonalize_fine");
}

int novak_selftest_orthogonalize_wait(const void *const *d_g, const int64_t *g_stride, int type, void *const *d_out,
                                      const int64_t *out_stride, const int64_t *rows, const int64_t *cols, int n,
                                      const double *coefficients, int steps, double eps, void *d_work,
                                      size_t work_bytes, int64_t withheld, uint64_t wait_ns, void *stream)
{
    OrthArgs a{d_g, g_stride, type, d_out, out_stride, rows, cols, n, {}, 0, eps, nullptr, nullptr, 0.0f, false, nullptr,
               0.0f, d_work, false, withheld, wait_ns};
    const char *where = "novak_selftest_orthogonalize_wait";
    if (withheld < 0) return orthogonalize(a, coefficients, steps, work_bytes, stream, where);
    // small matrices take the large ones' way, for which the caller's workspace has no place
    CHECK(check_orthogonalize(rows, cols, n, coefficients, steps, eps));
    const size_t need = orthogonalize_bytes(rows, cols, n, false, true);
    if (need == 0) return orthogonalize(a, coefficients, steps, work_bytes, stream, where);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    CHECK(finish(cudaMallocAsync(&a.work, need, s), where));
    const int rc = orthogonalize(a, coefficients, steps, need, stream, where), freed = finish(cudaFreeAsync(a.work, s), where);
    return rc != NOVAK_OK ? rc : freed;
}

int novak_orthogonal_step(float *const *d_theta, const void *const *d_g, int grad_type, float *const *d_m,
                          const int64_t *rows, const int64_t *cols, int n, double momentum, int nesterov,
                          const double *step, double decay, const double *coefficients, int steps, double eps,
                          void *d_work, size_t work_bytes, void *stream)
{
    return orthogonal_step(d_theta, d_g, grad_type, d_m, rows, cols, n, momentum, nesterov, step, decay, coefficients, steps, eps,
                           d_work, work_bytes, false, stream, "novak_orthogonal_step");
}

int novak_orthogonal_step_fine(float *const *d_theta, const void *const *d_g, int grad_type, float *const *d_m,
                               const int64_t *rows, const int64_t *cols, int n, double momentum, int nesterov,
                               const double *step, double decay, const double *coefficients, int steps, double eps,
                               void *d_work, size_t work_bytes, void *stream)
{
    return orthogonal_step(d_theta, d_g, grad_type, d_m, rows, cols, n, momentum, nesterov, step, decay, coefficients, steps, eps,
                           d_work, work_bytes, true, stream, "novak_orthogonal_step_fine");
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
