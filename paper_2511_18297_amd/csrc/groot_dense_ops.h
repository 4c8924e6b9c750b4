// The dense half of a network: grouped products, products in 8-bit integers, the AdamW step.  Host side and kernels.
#pragma once

#include "groot_internal.h"

namespace groot {

// One product over the groups of rows: out[i,:] = epilogue(A[i,:] B[g]) for the rows of every group.
struct RowsProduct {
    const void *A;               // [n, K], a_stride elements from row to row
    int64_t a_stride;
    const void *B;               // grouped products [groups, K, N] (b_n_major false) or [groups, N, K] (true)
    bool b_n_major;
    const int64_t *offsets;      // [groups + 1] or NULL
    const void *bias;            // [groups, N] or NULL
    const float *a_scale;        // 8-bit products: one per row
    const float *b_scale;        // ... [groups, N]
    bool relu;
    void *out;                   // [n, N]
    int64_t out_stride;
    int64_t n;
    int32_t groups, K, N;
};
// Kernel launchers: hipError_t as int, 0 = success; kErrTooManyTiles where a launch cannot hold them (2^32 lanes).
constexpr int kErrTooManyTiles = -4;
constexpr bool fits_launch(int64_t workgroups, int lanes) { return workgroups < ((int64_t)1 << 32) / lanes; }
int launch_grouped_rows(int32_t dtype, const RowsProduct &p, void *stream);
int launch_int8_rows(int32_t out_dtype, const RowsProduct &p, void *stream);
// the same for few rows of every group and weights [groups, N, K], where few_rows_serve says so (groot_few.hip)
bool few_rows_serve(const RowsProduct &p);
int launch_few_rows(int32_t dtype, const RowsProduct &p, void *stream);
int launch_few_int8(int32_t out_dtype, const RowsProduct &p, void *stream);
// ... of rows in floating point that are cut to 8 bits on the way (a_scale is not read)
bool few_linear_serves(const RowsProduct &p);
int launch_few_linear(int32_t dtype, const RowsProduct &p, void *stream);
int launch_quantize_rows(int32_t dtype, const void *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int64_t n,
                         int32_t K, void *stream);

// dW[g] = X_g^T dY_g and dbias[g] = column sums of dY_g
struct WeightsProduct {
    const void *X, *dY;
    int64_t x_stride, dy_stride;
    const int64_t *offsets;
    void *dW, *dbias;            // of dtype, or of float
    bool grad_f32;
    int64_t n;
    int32_t groups, K, N;
    void *workspace;
};
size_t grouped_weights_workspace(int32_t dtype, int64_t n, int32_t groups, int32_t K, int32_t N);
int launch_grouped_weights(int32_t dtype, const WeightsProduct &p, void *stream);

struct AdamwFactors {            // computed in fp64 and rounded once
    float decay, step_size, beta1, one_minus_beta1, beta2, one_minus_beta2, root_factor, eps;
};
constexpr int kAdamwBlock = 256;         // values that share a scale
int launch_adamw(const groot_adamw_tensor *tensors, int64_t n_tensors, int32_t param_dtype, int32_t grad_dtype, int32_t state_bits,
                 const AdamwFactors &f, const float *grad_scale, uint32_t step, uint32_t seed, void *stream);

struct RouteArgs {
    const void *scores;
    int64_t score_bytes;         // from row to row
    const float *bias;           // [E] or NULL
    int32_t *experts;            // [n, k]
    float *weights;              // [n, k]
    int32_t *places;             // [n, k]
    int64_t *offsets;            // [E + 1]
    int64_t n;
    int32_t dtype, E, k, gate, sets, open_sets, set_best;
    bool renormalise;
    bool by_value;               // the choice goes by probability + bias, not by the score
    double factor;
    // the launcher's
    int32_t rows;                // of a workgroup
    uint32_t inverse_k;
    int32_t set_lanes;           // lanes that hold a set, 0: it begins anywhere
    bool small_sets;             // a lane holds whole sets
    bool wide_sets;              // a lane's experts belong to two sets at the most
    int32_t value_bytes;         // of LDS for the sets
};
size_t route_workspace(int64_t n, int32_t E);
int launch_route(const RouteArgs &a, void *workspace, void *stream);

struct RouteBackwardArgs {
    const void *scores;
    int64_t score_bytes;
    const int32_t *experts;
    const float *dweights;
    void *dscores;
    int64_t ds_bytes;
    int64_t n;
    int32_t dtype, E, k, gate;
    bool renormalise;
    double factor;
};
int launch_route_backward(const RouteBackwardArgs &a, void *stream);

// rows at places[i, s] of R, which has `n_places` rows; a place outside is none
struct RoutedArgs {
    const void *X;               // [n, K]: rows to copy, or the gradient of the sum
    int64_t x_stride;            // elements
    const void *R;               // [n_places, K]
    int64_t r_stride;
    const int32_t *places;       // [n, k]
    const float *weights;        // [n, k] or NULL for ones
    const void *addend;          // [n, K] or NULL
    int64_t addend_stride;
    void *out;                   // [n, K], or [n_places, K]
    int64_t out_stride;
    const float *scale_in;       // [n] or NULL
    float *scale_out;            // [n_places]
    float *dweights;             // [n, k] or NULL
    int64_t n, n_places;
    int32_t k, K;
    int32_t part;                // pieces, or slots, of a row that a workgroup takes (the launcher's)
};
int launch_routed_rows(int32_t bytes, const RoutedArgs &a, void *stream);
int launch_routed_sum(int32_t dtype, const RoutedArgs &a, void *stream);
int launch_routed_sum_backward(int32_t dtype, const RoutedArgs &a, void *stream);

struct NormArgs {
    const void *X, *residual, *gain;         // residual, gain: or NULL
    void *H, *Y;                             // or NULL
    int8_t *Q;                               // or NULL
    float *q_scale, *rstd;                   // rstd: or NULL
    int64_t x_stride, residual_stride, h_stride, y_stride, q_stride;
    int64_t n;
    int32_t K;
    double eps;
};
int launch_norm(int32_t dtype, const NormArgs &a, void *stream);

struct NormBackwardArgs {
    const void *H, *gain, *dY, *dH;          // gain, dH: or NULL
    const float *rstd;
    void *dX, *dgain;                        // dgain: or NULL
    bool grad_f32;
    int64_t h_stride, dy_stride, dh_stride, dx_stride;
    int64_t n;
    int32_t K;
    float *partial;                          // [workgroups, K]
};
size_t norm_backward_workspace(int32_t dtype, int64_t n, int32_t K);
int launch_norm_backward(int32_t dtype, const NormBackwardArgs &a, void *stream);

}  // namespace groot
