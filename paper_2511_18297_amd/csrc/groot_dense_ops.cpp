// C entries of the grouped products, the products in 8-bit integers and the AdamW step: every argument is checked here, the
// kernels' launchers take what passed.
#include <cmath>

#include "groot_dense_ops.h"

using namespace groot;

namespace {

constexpr int32_t kMaxWidth = 65536, kMaxGroups = 65536;

int type_bytes(int32_t dtype)
{
    return dtype == GROOT_F32 ? 4 : dtype == GROOT_BF16 || dtype == GROOT_F16 ? 2 : 0;
}

bool aligned(const void *p, int to)
{
    return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0;
}

// [p, p + rows of `width` elements `stride` apart)
struct Span {
    const char *begin, *end;
    Span(const void *p, int64_t rows, int64_t stride, int64_t width, int bytes)
        : begin((const char *)p), end((const char *)p + (rows > 0 ? ((rows - 1) * stride + width) * bytes : 0)) {}
    bool meets(const Span &o) const { return begin < end && o.begin < o.end && begin < o.end && o.begin < end; }
};

groot_status bad(const char *who, const char *what)
{
    return fail(GROOT_EINVAL, std::string(who) + ": " + what);
}

groot_status launched(const char *who, int err)
{
    if (err == kErrTooManyTiles) return fail(GROOT_ERANGE, std::string(who) + ": more output tiles than a launch holds");
    return err ? fail(GROOT_EHIP, std::string(who) + ": launch failed: " + hip_error_text(err)) : GROOT_OK;
}

groot_status check_sizes(const char *who, int64_t n, int32_t groups, const int64_t *offsets, int32_t K, int32_t N)
{
    if (n < 0 || n > ((int64_t)1 << 40)) return bad(who, "n_rows must be in [0, 2^40]");
    if (K < 1 || K > kMaxWidth || N < 1 || N > kMaxWidth) return bad(who, "K and N must be in [1, 65536]");
    if (groups < 1 || groups > kMaxGroups) return bad(who, "n_groups must be in [1, 65536]");
    if (!offsets && groups != 1) return bad(who, "NULL offsets need n_groups = 1");
    if (!aligned(offsets, 8)) return bad(who, "offsets must be 8-byte aligned");
    return GROOT_OK;
}

groot_status check_matrix(const char *who, const char *name, const void *p, int64_t n, int64_t stride, int32_t width, int bytes)
{
    if (n > 0 && !p) return bad(who, (std::string(name) + " is NULL").c_str());
    if (!aligned(p, bytes)) return bad(who, (std::string(name) + " is not aligned to its type").c_str());
    if (stride < width || stride > ((int64_t)1 << 40)) return bad(who, (std::string(name) + ": the row stride is below the width").c_str());
    if (n > 0 && stride > (((int64_t)1 << 60) / n)) return bad(who, (std::string(name) + ": stride x rows is too large").c_str());
    return GROOT_OK;
}

}  // namespace

#define GROOT_TRY(call)                                                                                                                  \
    do {                                                                                                                                 \
        const groot_status st_ = (call);                                                                                                 \
        if (st_ != GROOT_OK) return st_;                                                                                                 \
    } while (0)

namespace {

// Y = act(X W + b), or with `transposed` dX = dY W^T; K: width of the input, N: of the output
groot_status rows_product(const char *who, int32_t dtype, const void *A, int64_t a_stride, const void *W, bool transposed,
                          const int64_t *offsets, const void *bias, int32_t relu, void *out, int64_t out_stride, int64_t n,
                          int32_t groups, int32_t K, int32_t N, void *stream)
{
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n, groups, offsets, K, N));
    GROOT_TRY(check_matrix(who, "the input", A, n, a_stride, K, b));
    GROOT_TRY(check_matrix(who, "the output", out, n, out_stride, N, b));
    if (!W) return bad(who, "W is NULL");
    if (!aligned(W, b) || !aligned(bias, b)) return bad(who, "W or bias is not aligned to its type");
    if (relu != 0 && relu != 1) return bad(who, "relu must be 0 or 1");
    const Span in(A, n, a_stride, K, b), to(out, n, out_stride, N, b), w(W, groups, (int64_t)K * N, (int64_t)K * N, b),
        bs(bias, bias ? groups : 0, N, N, b);
    if (to.meets(in) || to.meets(w) || to.meets(bs)) return bad(who, "the output overlaps an input");
    if (n == 0) return GROOT_OK;
    RowsProduct p{A, a_stride, W, transposed, offsets, bias, nullptr, nullptr, relu != 0, out, out_stride, n, groups, K, N};
    return launched(who, launch_grouped_rows(dtype, p, stream));
}

size_t quantized_stride(int32_t K) { return ((size_t)K + 15) / 16 * 16; }

groot_status check_int8(const char *who, const int8_t *W, const float *w_scale, const float *bias, int32_t relu, const void *Y,
                        int64_t y_stride, int64_t n, int32_t groups, int32_t K, int32_t N, int out_bytes)
{
    if (!W || !w_scale) return bad(who, "W or w_scale is NULL");
    if (!aligned(w_scale, 4) || !aligned(bias, 4)) return bad(who, "w_scale or bias is not aligned to its type");
    if (relu != 0 && relu != 1) return bad(who, "relu must be 0 or 1");
    const Span to(Y, n, y_stride, N, out_bytes), w(W, groups, (int64_t)K * N, (int64_t)K * N, 1), s(w_scale, groups, N, N, 4),
        bs(bias, bias ? groups : 0, N, N, 4);
    if (to.meets(w) || to.meets(s) || to.meets(bs)) return bad(who, "Y overlaps an input");
    return GROOT_OK;
}

}  // namespace

extern "C" groot_status groot_grouped_product(int32_t dtype, const void *X_dev, int64_t x_stride, const void *W_dev,
                                              const int64_t *offsets_dev, const void *bias_dev, int32_t relu, void *Y_dev,
                                              int64_t y_stride, int64_t n_rows, int32_t n_groups, int32_t K, int32_t N,
                                              void *hip_stream)
{
    return rows_product("groot_grouped_product", dtype, X_dev, x_stride, W_dev, false, offsets_dev, bias_dev, relu, Y_dev, y_stride,
                        n_rows, n_groups, K, N, hip_stream);
}

extern "C" groot_status groot_grouped_product_backward_data(int32_t dtype, const void *dY_dev, int64_t dy_stride, const void *W_dev,
                                                            const int64_t *offsets_dev, void *dX_dev, int64_t dx_stride,
                                                            int64_t n_rows, int32_t n_groups, int32_t K, int32_t N,
                                                            void *hip_stream)
{
    return rows_product("groot_grouped_product_backward_data", dtype, dY_dev, dy_stride, W_dev, true, offsets_dev, nullptr, 0, dX_dev,
                        dx_stride, n_rows, n_groups, N, K, hip_stream);
}

extern "C" groot_status groot_grouped_product_backward_weights_workspace(int32_t dtype, int64_t n_rows, int32_t n_groups, int32_t K,
                                                                         int32_t N, size_t *bytes)
{
    const char *who = "groot_grouped_product_backward_weights_workspace";
    if (!bytes) return bad(who, "bytes is NULL");
    if (!type_bytes(dtype)) return bad(who, "unknown dtype");
    const int64_t any = 0;
    GROOT_TRY(check_sizes(who, n_rows, n_groups, &any, K, N));
    *bytes = grouped_weights_workspace(dtype, n_rows, n_groups, K, N);
    return GROOT_OK;
}

extern "C" groot_status groot_grouped_product_backward_weights(int32_t dtype, const void *X_dev, int64_t x_stride,
                                                               const void *dY_dev, int64_t dy_stride, const int64_t *offsets_dev,
                                                               int32_t grad_dtype, void *dW_dev, void *dbias_dev, int64_t n_rows,
                                                               int32_t n_groups, int32_t K, int32_t N, void *workspace_dev,
                                                               size_t workspace_bytes, void *hip_stream)
{
    const char *who = "groot_grouped_product_backward_weights";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    if (grad_dtype != dtype && grad_dtype != GROOT_F32) return bad(who, "grad_dtype must be dtype or GROOT_F32");
    const int gb = type_bytes(grad_dtype);
    GROOT_TRY(check_sizes(who, n_rows, n_groups, offsets_dev, K, N));
    GROOT_TRY(check_matrix(who, "X", X_dev, n_rows, x_stride, K, b));
    GROOT_TRY(check_matrix(who, "dY", dY_dev, n_rows, dy_stride, N, b));
    if (!dW_dev) return bad(who, "dW is NULL");
    if (!aligned(dW_dev, gb) || !aligned(dbias_dev, gb)) return bad(who, "dW or dbias is not aligned to its type");
    const size_t need = grouped_weights_workspace(dtype, n_rows, n_groups, K, N);
    if (need && (!workspace_dev || workspace_bytes < need))
        return bad(who, "workspace too small (ask groot_grouped_product_backward_weights_workspace)");
    if (!aligned(workspace_dev, 16)) return bad(who, "the workspace must be 16-byte aligned");
    const Span x(X_dev, n_rows, x_stride, K, b), d(dY_dev, n_rows, dy_stride, N, b),
        w(dW_dev, n_groups, (int64_t)K * N, (int64_t)K * N, gb), s(dbias_dev, dbias_dev ? n_groups : 0, N, N, gb),
        ws(workspace_dev, need ? 1 : 0, (int64_t)need, (int64_t)need, 1);
    if (w.meets(x) || w.meets(d) || s.meets(x) || s.meets(d) || w.meets(s)) return bad(who, "an output overlaps an input or the other output");
    if (ws.meets(x) || ws.meets(d) || ws.meets(w) || ws.meets(s)) return bad(who, "the workspace overlaps a matrix");
    WeightsProduct p{X_dev, dY_dev, x_stride, dy_stride, offsets_dev, dW_dev, dbias_dev, grad_dtype == GROOT_F32, n_rows, n_groups, K, N,
                     workspace_dev};
    return launched(who, launch_grouped_weights(dtype, p, hip_stream));
}

extern "C" groot_status groot_quantize_rows(int32_t dtype, const void *X_dev, int64_t x_stride, int8_t *Q_dev, int64_t q_stride,
                                            float *scale_dev, int64_t n_rows, int32_t K, void *hip_stream)
{
    const char *who = "groot_quantize_rows";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n_rows, 1, nullptr, K, 1));
    GROOT_TRY(check_matrix(who, "X", X_dev, n_rows, x_stride, K, b));
    GROOT_TRY(check_matrix(who, "Q", Q_dev, n_rows, q_stride, K, 1));
    GROOT_TRY(check_matrix(who, "scale", scale_dev, n_rows, 1, 1, 4));
    const Span x(X_dev, n_rows, x_stride, K, b), q(Q_dev, n_rows, q_stride, K, 1), s(scale_dev, n_rows, 1, 1, 4);
    if (x.meets(q) || x.meets(s) || q.meets(s)) return bad(who, "two of X, Q and scale overlap");
    if (n_rows == 0) return GROOT_OK;
    return launched(who, launch_quantize_rows(dtype, X_dev, x_stride, Q_dev, q_stride, scale_dev, n_rows, K, hip_stream));
}

extern "C" groot_status groot_quantized_product(const int8_t *Q_dev, int64_t q_stride, const float *q_scale_dev, const int8_t *W_dev,
                                           const float *w_scale_dev, const int64_t *offsets_dev, const float *bias_dev, int32_t relu,
                                           int32_t dtype, void *Y_dev, int64_t y_stride, int64_t n_rows, int32_t n_groups, int32_t K,
                                           int32_t N, void *hip_stream)
{
    const char *who = "groot_quantized_product";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n_rows, n_groups, offsets_dev, K, N));
    GROOT_TRY(check_matrix(who, "Q", Q_dev, n_rows, q_stride, K, 1));
    GROOT_TRY(check_matrix(who, "q_scale", q_scale_dev, n_rows, 1, 1, 4));
    GROOT_TRY(check_matrix(who, "Y", Y_dev, n_rows, y_stride, N, b));
    GROOT_TRY(check_int8(who, W_dev, w_scale_dev, bias_dev, relu, Y_dev, y_stride, n_rows, n_groups, K, N, b));
    const Span to(Y_dev, n_rows, y_stride, N, b), q(Q_dev, n_rows, q_stride, K, 1), s(q_scale_dev, n_rows, 1, 1, 4);
    if (to.meets(q) || to.meets(s)) return bad(who, "Y overlaps an input");
    if (n_rows == 0) return GROOT_OK;
    RowsProduct p{Q_dev, q_stride, W_dev, true, offsets_dev, bias_dev, q_scale_dev, w_scale_dev, relu != 0, Y_dev, y_stride, n_rows,
                  n_groups, K, N};
    return launched(who, launch_int8_rows(dtype, p, hip_stream));
}

extern "C" groot_status groot_quantized_linear_workspace(int64_t n_rows, int32_t K, size_t *bytes)
{
    const char *who = "groot_quantized_linear_workspace";
    if (!bytes) return bad(who, "bytes is NULL");
    GROOT_TRY(check_sizes(who, n_rows, 1, nullptr, K, 1));
    *bytes = (size_t)n_rows * (quantized_stride(K) + 4);
    return GROOT_OK;
}

extern "C" groot_status groot_quantized_linear(int32_t dtype, const void *X_dev, int64_t x_stride, const int8_t *W_dev,
                                          const float *w_scale_dev, const int64_t *offsets_dev, const float *bias_dev, int32_t relu,
                                          void *Y_dev, int64_t y_stride, int64_t n_rows, int32_t n_groups, int32_t K, int32_t N,
                                          void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const char *who = "groot_quantized_linear";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n_rows, n_groups, offsets_dev, K, N));
    GROOT_TRY(check_matrix(who, "X", X_dev, n_rows, x_stride, K, b));
    GROOT_TRY(check_matrix(who, "Y", Y_dev, n_rows, y_stride, N, b));
    GROOT_TRY(check_int8(who, W_dev, w_scale_dev, bias_dev, relu, Y_dev, y_stride, n_rows, n_groups, K, N, b));
    const size_t row = quantized_stride(K), need = (size_t)n_rows * (row + 4);
    if (need && (!workspace_dev || workspace_bytes < need)) return bad(who, "workspace too small (ask groot_quantized_linear_workspace)");
    if (!aligned(workspace_dev, 16)) return bad(who, "the workspace must be 16-byte aligned");
    const Span to(Y_dev, n_rows, y_stride, N, b), x(X_dev, n_rows, x_stride, K, b), ws(workspace_dev, need ? 1 : 0, (int64_t)need, (int64_t)need, 1),
        w(W_dev, n_groups, (int64_t)K * N, (int64_t)K * N, 1), s(w_scale_dev, n_groups, N, N, 4), bs(bias_dev, bias_dev ? n_groups : 0, N, N, 4);
    if (to.meets(x)) return bad(who, "Y overlaps an input");
    if (ws.meets(to) || ws.meets(x) || ws.meets(w) || ws.meets(s) || ws.meets(bs)) return bad(who, "the workspace overlaps another argument");
    if (n_rows == 0) return GROOT_OK;
    RowsProduct x_rows{X_dev, x_stride, W_dev, true, offsets_dev, bias_dev, nullptr, w_scale_dev, relu != 0, Y_dev, y_stride, n_rows, n_groups, K, N};
    if (few_linear_serves(x_rows)) return launched(who, launch_few_linear(dtype, x_rows, hip_stream));
    int8_t *Q = (int8_t *)workspace_dev;
    float *scale = (float *)(Q + (size_t)n_rows * row);
    int err = launch_quantize_rows(dtype, X_dev, x_stride, Q, (int64_t)row, scale, n_rows, K, hip_stream);
    RowsProduct p{Q, (int64_t)row, W_dev, true, offsets_dev, bias_dev, scale, w_scale_dev, relu != 0, Y_dev, y_stride, n_rows, n_groups, K, N};
    if (!err) err = launch_int8_rows(dtype, p, hip_stream);
    return launched(who, err);
}

extern "C" groot_status groot_adamw_step(const groot_adamw_tensor *tensors, int64_t n_tensors, int32_t param_dtype, int32_t grad_dtype,
                                         int32_t state_bits, int64_t step, double lr, double beta1, double beta2, double eps,
                                         double weight_decay, const float *grad_scale_dev, uint32_t seed, void *hip_stream)
{
    const char *who = "groot_adamw_step";
    const int pb = type_bytes(param_dtype), gb = type_bytes(grad_dtype);
    if (!pb || !gb) return bad(who, "unknown dtype");
    if (state_bits != 8 && state_bits != 32) return bad(who, "state_bits must be 8 or 32");
    if (n_tensors < 0 || (n_tensors && !tensors)) return bad(who, "NULL tensors");
    if (step < 1) return bad(who, "step counts from 1");
    if (!(std::isfinite(lr) && lr >= 0) || !(std::isfinite(weight_decay) && weight_decay >= 0)) return bad(who, "lr and weight_decay must be finite and not negative");
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1)) return bad(who, "beta1 and beta2 must be in [0, 1)");
    if (!aligned(grad_scale_dev, 4)) return bad(who, "grad_scale is not aligned to its type");
    AdamwFactors f;
    f.decay = (float)(1.0 - lr * weight_decay);
    f.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    f.beta1 = (float)beta1;
    f.one_minus_beta1 = (float)(1.0 - beta1);
    f.beta2 = (float)beta2;
    f.one_minus_beta2 = (float)(1.0 - beta2);
    f.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    f.eps = (float)eps;
    // the factors that the kernel goes by: a denominator of 0 + 0, or 0 x infinity, would be NaN for values that nothing moves
    if (!(std::isfinite(f.eps) && f.eps > 0)) return bad(who, "eps must be finite and positive in fp32");
    if (!std::isfinite(f.step_size) || !std::isfinite(f.decay)) return bad(who, "lr / (1 - beta1^step) and 1 - lr weight_decay must be finite in fp32");
    const int sb = state_bits == 8 ? 1 : 4;
    bool master = false, first = true;
    for (int64_t t = 0; t < n_tensors; ++t) {
        const groot_adamw_tensor &x = tensors[t];
        if (x.n < 0) return bad(who, "a tensor's n is negative");
        if (x.n >= ((int64_t)1 << 33)) return fail(GROOT_ERANGE, std::string(who) + ": a tensor of 2^33 values or more");
        if (x.n == 0) continue;
        if (!x.param || !x.grad || !x.m || !x.v) return bad(who, "a tensor with a NULL array");
        if (state_bits == 8 && (!x.m_scale || !x.v_scale)) return bad(who, "8-bit states need m_scale and v_scale");
        if (!aligned(x.param, pb) || !aligned(x.grad, gb) || !aligned(x.m, sb) || !aligned(x.v, sb) || !aligned(x.master, 4) ||
            !aligned(x.m_scale, 4) || !aligned(x.v_scale, 4))
            return bad(who, "an array is not aligned to its type");
        if (!first && master != (x.master != nullptr)) return bad(who, "either all tensors have a master or none");
        master = x.master != nullptr;
        first = false;
    }
    if (first) return GROOT_OK;
    return launched(who, launch_adamw(tensors, n_tensors, param_dtype, grad_dtype, state_bits, f, grad_scale_dev, (uint32_t)step, seed,
                                      hip_stream));
}
