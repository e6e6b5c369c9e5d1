/*
 * ginex_layers.h - layers of a model on gathered rows: linear layers with bias, activation and residual, one for all rows
 * or one per expert, and the gradients of their rows and biases; a whole layer of experts for few rows; layer norm and the
 * lookup of learned rows with their gradients.  Conventions are those of ginex_train.h: device pointers unless marked host,
 * the caller owns every buffer, 0 or a negative GINEX_ERR_* code, arguments checked on the host before anything is launched,
 * calls that only enqueue on `stream`, allocate nothing and may be captured; what a call writes may not overlap its other
 * arrays unless it says so, and calls that may run at the same time need a workspace each.  Equal inputs give equal bits.
 */
#ifndef GINEX_LAYERS_H
#define GINEX_LAYERS_H

#include "ginex_train.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GINEX_MAX_FEW_ROWS 64 /* rows of ginex_expert_layer */
#define GINEX_MAX_FEW_TOP 16  /* and its choices a row */

/* The weights of one linear layer per expert: element (e, c, d), c < width, d < out, is
 * data[e * expert_stride + c * stride + d], or, turned, data[e * expert_stride + d * stride + c].  Aligned to the type. */
typedef struct ginex_weights {
  const void* data;
  int32_t experts;       /* 1 .. GINEX_MAX_EXPERTS */
  int32_t turned;        /* 0: d is dense; 1: c is */
  int64_t width;         /* 1 .. GINEX_MAX_WIDTH */
  int64_t out;           /* 1 .. GINEX_MAX_WIDTH */
  int64_t stride;        /* 0, or at least the dense size; below 2^31 */
  int64_t expert_stride; /* 0 or more */
  int32_t type;          /* GINEX_F32, _BF16, _F16 */
} ginex_weights_t;

/* y[s, :] = f(x[s, :] W + bias) + residual[s, :], products summed in f32, the rest in f32, rounded once.  f32 factors may be
 * taken as three bf16 each: a product is then good to 2^-24 of itself, as a rounded one is, and what a factor has below 2^-133
 * is left out.  bias [experts x out], of x's type, may be NULL (0), and so may residual.  Without a route s is a row,
 * weights->experts is 1.  With one s is a slot, W and bias are its expert's, and x[s] is x[source[s]] (by_slot 0; x has `rows`
 * rows) or x[s] itself (by_slot 1; rows * top); a slot without a row counts as a row of zeros, and y's rows from
 * offsets[experts] on are cleared.  kept not NULL: what f is applied to, in 8 bits (for ginex_activate_backward); cleared rows
 * are codes of 0.  y may be residual. */
int32_t ginex_linear(const ginex_rows_t* x /*host struct*/, const ginex_weights_t* weights /*host struct*/, const void* bias,
                     int32_t activation, const ginex_rows_t* residual /*host struct or NULL*/,
                     const ginex_routing_t* route /*host struct or NULL*/, int32_t by_slot,
                     const ginex_rows_t* y /*host struct*/, const ginex_codes_t* kept /*host struct or NULL*/, void* stream);

/* The gradient of the bias: dbias[e, :] = sum over the slots s of expert e of dy[s, :], f32, 0 for an expert without rows;
 * route NULL: one sum over all rows. */
size_t ginex_bias_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width);

int32_t ginex_bias_gradient(const ginex_rows_t* dy /*host struct*/, const ginex_routing_t* route /*host struct or NULL*/,
                            float* dbias, void* ws, size_t ws_bytes, void* stream);

/* A layer of experts for up to GINEX_MAX_FEW_ROWS rows: y[r, :] = sum over j < top of p(r, j) f(x[r, :] W_e + bias_e), where
 * e = e(r, 0), e(r, 1), .. are the experts of the largest <x[r, :], router[e, :]>, of equal ones the first, and p(r, :) is the
 * softmax over those.  Scores are sums in f64 (what is chosen should not hang on an order of f32
 * sums), the rest is f32, rounded once.  A NaN
 * counts as larger than any number, and leaves NaN.  router has a row of x's width for each of the experts; top is at most
 * their number and GINEX_MAX_FEW_TOP. */
size_t ginex_expert_layer_workspace_bytes(int64_t rows, int32_t top, int32_t experts, int64_t width, int64_t out);

int32_t ginex_expert_layer(const ginex_rows_t* x /*host struct*/, const ginex_rows_t* router /*host struct*/,
                           const ginex_weights_t* weights /*host struct*/, const void* bias, int32_t top,
                           int32_t activation, const ginex_rows_t* y /*host struct*/, void* ws, size_t ws_bytes,
                           void* stream);

/* y[r, :] = (x[r, :] - mean) * rstd * weight + bias, mean and rstd = 1 / sqrt(variance + eps) of the row in f32, variance
 * the mean of the squared distances from the mean; rounded once.  weight and bias [width], of x's type, may be NULL (1, 0).
 * stats, not NULL: f32 [rows x 2], mean and rstd of every row.  eps >= 0.  y may be x. */
int32_t ginex_layer_norm(const ginex_rows_t* x /*host struct*/, const void* weight, const void* bias, float eps,
                         const ginex_rows_t* y /*host struct*/, float* stats, void* stream);

/* With unit = (x - mean) rstd and a = dy weight: dx[r, :] = rstd (a - mean(a) - unit mean(a unit)), means over the row;
 * dweight = sum over the rows of dy unit and dbias = that of dy, f32 [width] (both NULL: left out).  dx may be dy. */
size_t ginex_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width);

int32_t ginex_layer_norm_backward(const ginex_rows_t* dy /*host struct*/, const ginex_rows_t* x /*host struct*/,
                                  const float* stats, const void* weight, const ginex_rows_t* dx /*host struct*/,
                                  float* dweight, float* dbias, void* ws, size_t ws_bytes, void* stream);

/* out[i, :] = scale * table[ids[i], :], rounded once; 0 where ids[i] is no row of the table.  ids are int32 (ids_64 = 0) or
 * int64 (1), as many as out has rows. */
int32_t ginex_lookup(const ginex_rows_t* table /*host struct*/, const void* ids, int32_t ids_64, float scale,
                     const ginex_rows_t* out /*host struct*/, void* stream);

/* The table's gradient: dtable[v, :] = scale * sum over the i with ids[i] = v of dy[i, :], the sum in f32 in an order that
 * depends on the ids alone, rounded once; 0 for a row that no id names.  Up to 2^30 ids. */
size_t ginex_lookup_backward_workspace_bytes(int64_t ids, int64_t rows, int64_t width);

int32_t ginex_lookup_backward(const ginex_rows_t* dy /*host struct*/, const void* ids, int32_t ids_64, float scale,
                              const ginex_rows_t* dtable /*host struct*/, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GINEX_LAYERS_H */
