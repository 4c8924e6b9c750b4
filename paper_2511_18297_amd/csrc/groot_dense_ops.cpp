// C entries of the grouped products, the products in 8-bit integers, the AdamW step, the routing and the norm: every argument is
// checked here, the kernels' launchers take what passed.
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

namespace {

constexpr int32_t kMaxExperts = 1024, kMaxTopK = 32, kMaxSets = 64;
constexpr int64_t kMaxSlots = ((int64_t)1 << 31) - 1;

groot_status check_gate(const char *who, int64_t n, int32_t E, int32_t k, int32_t gate, int32_t renormalise, double factor)
{
    if (E < 1 || E > kMaxExperts) return bad(who, "n_experts must be in [1, 1024]");
    if (k < 1 || k > kMaxTopK || k > E) return bad(who, "top_k must be in [1, 32] and at most n_experts");
    if (n < 0) return bad(who, "n_rows must not be negative");
    if (n > kMaxSlots / k) return fail(GROOT_ERANGE, std::string(who) + ": 2^31 slots or more");
    if (gate != GROOT_SOFTMAX && gate != GROOT_SIGMOID) return bad(who, "unknown gate");
    if (renormalise != 0 && renormalise != 1) return bad(who, "renormalise must be 0 or 1");
    if (!std::isfinite(factor) || !std::isfinite((float)factor)) return bad(who, "factor must be finite in fp32");
    return GROOT_OK;
}

// rows, their places and the matrix that these name
groot_status check_routed(const char *who, int64_t n, int32_t k, int64_t n_places, int32_t K, const int32_t *places)
{
    if (k < 1 || k > kMaxTopK) return bad(who, "top_k must be in [1, 32]");
    if (n < 0 || n_places < 0) return bad(who, "n_rows and n_places must not be negative");
    if (n > kMaxSlots / k || n_places > kMaxSlots) return fail(GROOT_ERANGE, std::string(who) + ": 2^31 slots or places or more");
    if (K < 1 || K > kMaxWidth) return bad(who, "width must be in [1, 65536]");
    return check_matrix(who, "places", places, n, k, k, 4);
}

// an output that is a matrix given as input, element for element, or apart from it
bool same_or_apart(const Span &out, const Span &in, int64_t out_stride, int64_t in_stride, int64_t n)
{
    return !out.meets(in) || (out.begin == in.begin && (out_stride == in_stride || n <= 1));
}

}  // namespace

extern "C" groot_status groot_route_workspace(int64_t n_rows, int32_t n_experts, int32_t top_k, size_t *bytes)
{
    const char *who = "groot_route_workspace";
    if (!bytes) return bad(who, "bytes is NULL");
    GROOT_TRY(check_gate(who, n_rows, n_experts, top_k, GROOT_SOFTMAX, 0, 1.0));
    *bytes = route_workspace(n_rows, n_experts);
    return GROOT_OK;
}

extern "C" groot_status groot_route(int32_t dtype, const void *scores_dev, int64_t score_stride, const float *bias_dev, int32_t gate,
                                    int32_t n_sets, int32_t open_sets, int32_t set_best, int32_t renormalise, double factor,
                                    int32_t *experts_dev, float *weights_dev, int32_t *places_dev, int64_t *offsets_dev, int64_t n_rows,
                                    int32_t n_experts, int32_t top_k, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const char *who = "groot_route";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_gate(who, n_rows, n_experts, top_k, gate, renormalise, factor));
    if (n_sets < 1 || n_sets > kMaxSets || n_experts % n_sets) return bad(who, "n_sets must be in [1, 64] and divide n_experts");
    if (open_sets < 1 || open_sets > n_sets) return bad(who, "open_sets must be in [1, n_sets]");
    if (set_best < 1 || set_best > 2 || set_best > n_experts / n_sets) return bad(who, "set_best must be 1 or 2 and at most a set's experts");
    if (top_k > open_sets * (n_experts / n_sets)) return bad(who, "top_k is more than the open sets hold");
    GROOT_TRY(check_matrix(who, "scores", scores_dev, n_rows, score_stride, n_experts, b));
    GROOT_TRY(check_matrix(who, "experts", experts_dev, n_rows, top_k, top_k, 4));
    GROOT_TRY(check_matrix(who, "weights", weights_dev, n_rows, top_k, top_k, 4));
    GROOT_TRY(check_matrix(who, "places", places_dev, n_rows, top_k, top_k, 4));
    if (!offsets_dev || !aligned(offsets_dev, 8)) return bad(who, "offsets must be given and 8-byte aligned");
    if (!aligned(bias_dev, 4)) return bad(who, "bias is not aligned to its type");
    const size_t need = route_workspace(n_rows, n_experts);
    if (need && (!workspace_dev || workspace_bytes < need)) return bad(who, "workspace too small (ask groot_route_workspace)");
    if (!aligned(workspace_dev, 16)) return bad(who, "the workspace must be 16-byte aligned");
    const Span in(scores_dev, n_rows, score_stride, n_experts, b), bs(bias_dev, bias_dev ? 1 : 0, n_experts, n_experts, 4),
        out[] = {Span(experts_dev, n_rows, top_k, top_k, 4), Span(weights_dev, n_rows, top_k, top_k, 4), Span(places_dev, n_rows, top_k, top_k, 4),
                 Span(offsets_dev, 1, n_experts + 1, n_experts + 1, 8), Span(workspace_dev, need ? 1 : 0, (int64_t)need, (int64_t)need, 1)};
    for (int i = 0; i < 5; ++i) {
        if (out[i].meets(in) || out[i].meets(bs)) return bad(who, "an output or the workspace overlaps an input");
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return bad(who, "two of the outputs and the workspace overlap");
    }
    RouteArgs a{scores_dev, score_stride * b, bias_dev, experts_dev, weights_dev, places_dev, offsets_dev, n_rows, dtype, n_experts, top_k, gate,
                n_sets, open_sets, set_best, renormalise != 0, bias_dev != nullptr || (set_best == 2 && open_sets < n_sets), factor, 0, 0, 0, false, false, 0};
    return launched(who, launch_route(a, workspace_dev, hip_stream));
}

extern "C" groot_status groot_route_backward(int32_t dtype, const void *scores_dev, int64_t score_stride, int32_t gate, int32_t renormalise,
                                             double factor, const int32_t *experts_dev, const float *dweights_dev, void *dscores_dev,
                                             int64_t ds_stride, int64_t n_rows, int32_t n_experts, int32_t top_k, void *hip_stream)
{
    const char *who = "groot_route_backward";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_gate(who, n_rows, n_experts, top_k, gate, renormalise, factor));
    GROOT_TRY(check_matrix(who, "scores", scores_dev, n_rows, score_stride, n_experts, b));
    GROOT_TRY(check_matrix(who, "dscores", dscores_dev, n_rows, ds_stride, n_experts, b));
    GROOT_TRY(check_matrix(who, "experts", experts_dev, n_rows, top_k, top_k, 4));
    GROOT_TRY(check_matrix(who, "dweights", dweights_dev, n_rows, top_k, top_k, 4));
    const Span to(dscores_dev, n_rows, ds_stride, n_experts, b), in(scores_dev, n_rows, score_stride, n_experts, b),
        e(experts_dev, n_rows, top_k, top_k, 4), d(dweights_dev, n_rows, top_k, top_k, 4);
    if (to.meets(in) || to.meets(e) || to.meets(d)) return bad(who, "dscores overlaps an input");
    if (n_rows == 0) return GROOT_OK;
    RouteBackwardArgs a{scores_dev, score_stride * b, experts_dev, dweights_dev, dscores_dev, ds_stride * b, n_rows, dtype, n_experts, top_k, gate,
                        renormalise != 0, factor};
    return launched(who, launch_route_backward(a, hip_stream));
}

extern "C" groot_status groot_routed_rows(int32_t dtype, const void *X_dev, int64_t x_stride, const float *x_scale_dev, const int32_t *places_dev,
                                          int32_t top_k, void *R_dev, int64_t r_stride, float *r_scale_dev, int64_t n_rows, int64_t n_places,
                                          int32_t width, void *hip_stream)
{
    const char *who = "groot_routed_rows";
    const int b = dtype == GROOT_I8 ? 1 : type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_routed(who, n_rows, top_k, n_places, width, places_dev));
    GROOT_TRY(check_matrix(who, "X", X_dev, n_rows, x_stride, width, b));
    GROOT_TRY(check_matrix(who, "R", R_dev, n_places, r_stride, width, b));
    const bool scaled = x_scale_dev != nullptr || r_scale_dev != nullptr;
    if (scaled) {
        GROOT_TRY(check_matrix(who, "x_scale", x_scale_dev, n_rows, 1, 1, 4));
        GROOT_TRY(check_matrix(who, "r_scale", r_scale_dev, n_places, 1, 1, 4));
    }
    const Span x(X_dev, n_rows, x_stride, width, b), r(R_dev, n_places, r_stride, width, b), p(places_dev, n_rows, top_k, top_k, 4),
        xs(x_scale_dev, scaled ? n_rows : 0, 1, 1, 4), rs(r_scale_dev, scaled ? n_places : 0, 1, 1, 4);
    if (r.meets(x) || r.meets(p) || r.meets(xs) || rs.meets(x) || rs.meets(p) || rs.meets(xs) || r.meets(rs)) return bad(who, "an output overlaps an input or the other output");
    if (n_rows == 0 || n_places == 0) return GROOT_OK;
    RoutedArgs a{};
    a.X = X_dev, a.x_stride = x_stride, a.places = places_dev, a.out = R_dev, a.out_stride = r_stride;
    a.scale_in = x_scale_dev, a.scale_out = r_scale_dev, a.n = n_rows, a.n_places = n_places, a.k = top_k, a.K = width;
    return launched(who, launch_routed_rows(b, a, hip_stream));
}

extern "C" groot_status groot_routed_sum(int32_t dtype, const void *R_dev, int64_t r_stride, const int32_t *places_dev, const float *weights_dev,
                                         const void *addend_dev, int64_t addend_stride, int32_t top_k, void *out_dev, int64_t out_stride,
                                         int64_t n_rows, int64_t n_places, int32_t width, void *hip_stream)
{
    const char *who = "groot_routed_sum";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_routed(who, n_rows, top_k, n_places, width, places_dev));
    GROOT_TRY(check_matrix(who, "R", R_dev, n_places, r_stride, width, b));
    GROOT_TRY(check_matrix(who, "out", out_dev, n_rows, out_stride, width, b));
    if (addend_dev) GROOT_TRY(check_matrix(who, "addend", addend_dev, n_rows, addend_stride, width, b));
    if (!aligned(weights_dev, 4)) return bad(who, "weights is not aligned to its type");
    const Span to(out_dev, n_rows, out_stride, width, b), r(R_dev, n_places, r_stride, width, b), p(places_dev, n_rows, top_k, top_k, 4),
        w(weights_dev, weights_dev ? n_rows : 0, top_k, top_k, 4), add(addend_dev, addend_dev ? n_rows : 0, addend_stride, width, b);
    if (to.meets(r) || to.meets(p) || to.meets(w)) return bad(who, "out overlaps an input");
    if (to.meets(add)) return bad(who, "out overlaps addend");
    if (n_rows == 0) return GROOT_OK;
    RoutedArgs a{};
    a.R = R_dev, a.r_stride = r_stride, a.places = places_dev, a.weights = weights_dev, a.addend = addend_dev, a.addend_stride = addend_stride;
    a.out = out_dev, a.out_stride = out_stride, a.n = n_rows, a.n_places = n_places, a.k = top_k, a.K = width;
    return launched(who, launch_routed_sum(dtype, a, hip_stream));
}

extern "C" groot_status groot_routed_sum_backward(int32_t dtype, const void *dout_dev, int64_t dout_stride, const void *R_dev, int64_t r_stride,
                                                  const int32_t *places_dev, const float *weights_dev, int32_t top_k, void *dR_dev,
                                                  int64_t dr_stride, float *dweights_dev, int64_t n_rows, int64_t n_places, int32_t width,
                                                  void *hip_stream)
{
    const char *who = "groot_routed_sum_backward";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_routed(who, n_rows, top_k, n_places, width, places_dev));
    GROOT_TRY(check_matrix(who, "dout", dout_dev, n_rows, dout_stride, width, b));
    if (n_rows > 0 && n_places > 0 && !dR_dev && !dweights_dev) return bad(who, "dR and dweights are both NULL");
    if (dweights_dev) GROOT_TRY(check_matrix(who, "R", R_dev, n_places, r_stride, width, b));
    if (dR_dev) GROOT_TRY(check_matrix(who, "dR", dR_dev, n_places, dr_stride, width, b));
    if (!aligned(weights_dev, 4) || !aligned(dweights_dev, 4)) return bad(who, "weights or dweights is not aligned to its type");
    const Span dr(dR_dev, dR_dev ? n_places : 0, dr_stride, width, b), dw(dweights_dev, dweights_dev ? n_rows : 0, top_k, top_k, 4),
        d(dout_dev, n_rows, dout_stride, width, b), r(R_dev, dweights_dev ? n_places : 0, r_stride, width, b),
        p(places_dev, n_rows, top_k, top_k, 4), w(weights_dev, weights_dev ? n_rows : 0, top_k, top_k, 4);
    if (dr.meets(d) || dr.meets(r) || dr.meets(p) || dr.meets(w) || dw.meets(d) || dw.meets(r) || dw.meets(p) || dw.meets(w) || dr.meets(dw))
        return bad(who, "an output overlaps an input or the other output");
    if (n_rows == 0) return GROOT_OK;
    RoutedArgs a{};
    a.X = dout_dev, a.x_stride = dout_stride, a.R = R_dev, a.r_stride = r_stride, a.places = places_dev, a.weights = weights_dev;
    a.out = dR_dev, a.out_stride = dr_stride, a.dweights = dweights_dev, a.n = n_rows, a.n_places = n_places, a.k = top_k, a.K = width;
    return launched(who, launch_routed_sum_backward(dtype, a, hip_stream));
}

extern "C" groot_status groot_rms_norm(int32_t dtype, const void *X_dev, int64_t x_stride, const void *residual_dev, int64_t residual_stride,
                                       const void *gain_dev, double eps, void *H_dev, int64_t h_stride, void *Y_dev, int64_t y_stride,
                                       int8_t *Q_dev, int64_t q_stride, float *q_scale_dev, float *rstd_dev, int64_t n_rows, int32_t width,
                                       void *hip_stream)
{
    const char *who = "groot_rms_norm";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n_rows, 1, nullptr, width, 1));
    if (!std::isfinite((float)eps) || !((float)eps > 0)) return bad(who, "eps must be finite and positive in fp32");
    GROOT_TRY(check_matrix(who, "X", X_dev, n_rows, x_stride, width, b));
    if (residual_dev) GROOT_TRY(check_matrix(who, "residual", residual_dev, n_rows, residual_stride, width, b));
    if (H_dev) GROOT_TRY(check_matrix(who, "H", H_dev, n_rows, h_stride, width, b));
    if (Y_dev) GROOT_TRY(check_matrix(who, "Y", Y_dev, n_rows, y_stride, width, b));
    if ((Q_dev != nullptr) != (q_scale_dev != nullptr)) return bad(who, "Q and q_scale go together");
    if (Q_dev) GROOT_TRY(check_matrix(who, "Q", Q_dev, n_rows, q_stride, width, 1));
    if (n_rows > 0 && !Y_dev && !Q_dev && !H_dev && !rstd_dev) return bad(who, "no output is asked for");
    if (!aligned(gain_dev, b) || !aligned(q_scale_dev, 4) || !aligned(rstd_dev, 4)) return bad(who, "gain, q_scale or rstd is not aligned to its type");
    const Span x(X_dev, n_rows, x_stride, width, b), r(residual_dev, residual_dev ? n_rows : 0, residual_stride, width, b),
        g(gain_dev, gain_dev ? 1 : 0, width, width, b);
    const Span out[] = {Span(H_dev, H_dev ? n_rows : 0, h_stride, width, b), Span(Y_dev, Y_dev ? n_rows : 0, y_stride, width, b),
                        Span(Q_dev, Q_dev ? n_rows : 0, q_stride, width, 1), Span(q_scale_dev, q_scale_dev ? n_rows : 0, 1, 1, 4),
                        Span(rstd_dev, rstd_dev ? n_rows : 0, 1, 1, 4)};
    const int64_t strides[] = {h_stride, y_stride};
    for (int i = 0; i < 5; ++i) {
        // H and Y may take the place of an input, row for row: a row is read whole before any of it is written
        if (i < 2 ? !same_or_apart(out[i], x, strides[i], x_stride, n_rows) || !same_or_apart(out[i], r, strides[i], residual_stride, n_rows)
                  : out[i].meets(x) || out[i].meets(r))
            return bad(who, "an output overlaps an input that it is not the same matrix as");
        if (out[i].meets(g)) return bad(who, "an output overlaps gain");
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return bad(who, "two outputs overlap");
    }
    if (n_rows == 0) return GROOT_OK;
    NormArgs a{X_dev, residual_dev, gain_dev, H_dev, Y_dev, Q_dev, q_scale_dev, rstd_dev, x_stride, residual_stride, h_stride, y_stride, q_stride,
               n_rows, width, eps};
    return launched(who, launch_norm(dtype, a, hip_stream));
}

extern "C" groot_status groot_rms_norm_backward_workspace(int32_t dtype, int64_t n_rows, int32_t width, size_t *bytes)
{
    const char *who = "groot_rms_norm_backward_workspace";
    if (!bytes) return bad(who, "bytes is NULL");
    if (!type_bytes(dtype)) return bad(who, "unknown dtype");
    GROOT_TRY(check_sizes(who, n_rows, 1, nullptr, width, 1));
    *bytes = norm_backward_workspace(dtype, n_rows, width);
    return GROOT_OK;
}

extern "C" groot_status groot_rms_norm_backward(int32_t dtype, const void *H_dev, int64_t h_stride, const float *rstd_dev, const void *gain_dev,
                                                const void *dY_dev, int64_t dy_stride, const void *dH_dev, int64_t dh_stride, void *dX_dev,
                                                int64_t dx_stride, int32_t grad_dtype, void *dgain_dev, int64_t n_rows, int32_t width,
                                                void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const char *who = "groot_rms_norm_backward";
    const int b = type_bytes(dtype);
    if (!b) return bad(who, "unknown dtype");
    if (grad_dtype != dtype && grad_dtype != GROOT_F32) return bad(who, "grad_dtype must be dtype or GROOT_F32");
    const int gb = type_bytes(grad_dtype);
    GROOT_TRY(check_sizes(who, n_rows, 1, nullptr, width, 1));
    GROOT_TRY(check_matrix(who, "H", H_dev, n_rows, h_stride, width, b));
    GROOT_TRY(check_matrix(who, "rstd", rstd_dev, n_rows, 1, 1, 4));
    GROOT_TRY(check_matrix(who, "dY", dY_dev, n_rows, dy_stride, width, b));
    if (dH_dev) GROOT_TRY(check_matrix(who, "dH", dH_dev, n_rows, dh_stride, width, b));
    GROOT_TRY(check_matrix(who, "dX", dX_dev, n_rows, dx_stride, width, b));
    if (!aligned(gain_dev, b) || !aligned(dgain_dev, gb)) return bad(who, "gain or dgain is not aligned to its type");
    const size_t need = dgain_dev ? norm_backward_workspace(dtype, n_rows, width) : 0;
    if (need && (!workspace_dev || workspace_bytes < need)) return bad(who, "workspace too small (ask groot_rms_norm_backward_workspace)");
    if (!aligned(workspace_dev, 16)) return bad(who, "the workspace must be 16-byte aligned");
    const Span in[] = {Span(H_dev, n_rows, h_stride, width, b), Span(rstd_dev, n_rows, 1, 1, 4), Span(gain_dev, gain_dev ? 1 : 0, width, width, b),
                       Span(dY_dev, n_rows, dy_stride, width, b), Span(dH_dev, dH_dev ? n_rows : 0, dh_stride, width, b)},
        out[] = {Span(dX_dev, n_rows, dx_stride, width, b), Span(dgain_dev, dgain_dev ? 1 : 0, width, width, gb),
                 Span(workspace_dev, need ? 1 : 0, (int64_t)need, (int64_t)need, 1)};
    for (int i = 0; i < 3; ++i) {
        for (const Span &s : in)
            if (out[i].meets(s)) return bad(who, "an output or the workspace overlaps an input");
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return bad(who, "two of the outputs and the workspace overlap");
    }
    if (n_rows == 0 && !dgain_dev) return GROOT_OK;
    NormBackwardArgs a{H_dev, gain_dev, dY_dev, dH_dev, rstd_dev, dX_dev, dgain_dev, grad_dtype == GROOT_F32, h_stride, dy_stride, dh_stride,
                       dx_stride, n_rows, width, (float *)workspace_dev};
    return launched(who, launch_norm_backward(dtype, a, hip_stream));
}
