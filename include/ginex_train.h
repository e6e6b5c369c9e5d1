/*
 * ginex_train.h - operators of the training step that consumes the gathered rows: rows sorted by
 * expert and back (with the gradients of both), and activations kept in 8 bits with their use in
 * the backward pass.  Conventions are those of ginex.h: device pointers unless marked host, the
 * caller owns every buffer, 0 or a negative GINEX_ERR_* code, ginex_last_error(), arguments checked
 * on the host before anything is launched.  Every call here only enqueues on `stream`, allocates
 * nothing and may be captured into a graph; what it writes may not overlap its other arrays unless it
 * says so.  Equal inputs give equal bits: nothing here depends on the order in which workgroups run.
 */
#ifndef GINEX_TRAIN_H
#define GINEX_TRAIN_H

#include "ginex.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of the elements of rows. */
#define GINEX_F32 0
#define GINEX_BF16 1
#define GINEX_F16 2

#define GINEX_ACT_NONE 0
#define GINEX_ACT_RELU 1 /* x < 0 ? 0 : x */
#define GINEX_ACT_SILU 2 /* x / (1 + exp(-x)) */
#define GINEX_ACT_GELU 3 /* x * Phi(x), Phi the normal distribution function (no approximation by tanh) */
/* Both and their derivatives are computed in f32 and rounded once.  Of rows in f32 silu is good to 2^-20 of its value and gelu
 * to 2^-18 + x^2 2^-22 of it; of rows in 16 bits exp and 1/x are the hardware's (1 unit each, exp's argument rounded) and Phi
 * is good to 2^-19 + x^2 2^-23 of it, below the rounding of the result.  Results below 2^-119 may be 0. */

#define GINEX_MAX_EXPERTS 1024
#define GINEX_MAX_TOP 64
#define GINEX_MAX_WIDTH (1 << 20)
#define GINEX_CODE_BLOCK 32 /* channels that share a scale */

/* A matrix of rows in HBM: element (r, c) is data[r * stride + c], aligned to its type.  Rows need not
 * be aligned to more than that; vectors of 16 bytes are read and written at any such address.  Rows that
 * are only read may overlap (stride 0: one row for all); rows that are written may not. */
typedef struct ginex_rows {
  void* data;
  int64_t rows;
  int64_t width;  /* 1 .. GINEX_MAX_WIDTH elements */
  int64_t stride; /* elements from a row to the next: 0 or at least width (written rows: at least width) */
  int32_t type;   /* GINEX_F32, _BF16, _F16 */
} ginex_rows_t;

/* Where rows go.  Row r has `top` choices of an expert; pair (r, j) is in slot slot[r * top + j], or in
 * none (-1).  The slots of expert e are offsets[e] .. offsets[e+1] - 1, from offsets[0] = 0 on and ascending, its
 * rows in ascending order of (r, j); source[s] is the row in slot s, -1 for the slots from offsets[experts] on.
 * Arrays that hold anything else give results without meaning, but nothing outside the arrays is read or
 * written for them. */
typedef struct ginex_routing {
  int64_t rows;
  int32_t top;      /* 1 .. GINEX_MAX_TOP; rows * top < 2^31 */
  int32_t experts;  /* 1 .. GINEX_MAX_EXPERTS */
  int64_t* offsets; /* [experts + 1] */
  int32_t* slot;    /* [rows * top] */
  int32_t* source;  /* [rows * top] */
} ginex_routing_t;

/* Rows in 8 bits (the INT8 format of the OCP Microscaling specification 1.0: 32 values that share a
 * power of two).  With b = ceil(width / 32) blocks a row, codes is [rows x 32 b] and scales [rows x b].
 * A block's e is floor(log2(its largest magnitude)), -120 at least; a value x is kept as
 * q = clamp(round(x * 2^(6 - e)), -127, 127), halves to even, and stands for q * 2^(e - 6); the scale
 * byte is e + 127.  A block that held an infinity or a NaN has scale byte 255 and stands for NaN.  Codes
 * behind the width are 0 and do not count.
 * codes are aligned to 8 bytes. */
typedef struct ginex_codes {
  int64_t rows;
  int64_t width;
  int8_t* codes;
  uint8_t* scales;
} ginex_codes_t;

/* Sorts pairs by expert (a stable sort: equal experts keep the order of (r, j)).  `chosen` [rows * top]
 * holds the experts as int32 (chosen_64 = 0) or int64 (1); a value outside [0, experts) means no expert.
 * capacity: most slots of an expert, the first of its pairs get them; negative = no bound.  The arrays
 * that `out` points to are written.  rows may be 0. */
size_t ginex_route_workspace_bytes(int64_t rows, int32_t top, int32_t experts);

int32_t ginex_route(const void* chosen, int32_t chosen_64, int64_t capacity,
                    const ginex_routing_t* out /*host struct*/, void* ws, size_t ws_bytes, void* stream);

/* out[slot[r * top + j], :] = x[r, :] for every pair that has a slot; the rows of `out` from
 * offsets[experts] on are cleared.  x has `rows` rows, out rows * top. */
int32_t ginex_dispatch(const ginex_routing_t* route /*host struct*/, const ginex_rows_t* x /*host struct*/,
                       const ginex_rows_t* out /*host struct*/, void* stream);

/* y[r, :] = sum over j of weights[r * top + j] * z[slot[r * top + j], :], in f32 and in the order of j,
 * rounded once; pairs without a slot do not count, whatever their weight.  weights NULL: all 1, which
 * makes it the gradient of ginex_dispatch. */
int32_t ginex_combine(const ginex_routing_t* route /*host struct*/, const ginex_rows_t* z /*host struct*/,
                      const float* weights, const ginex_rows_t* y /*host struct*/, void* stream);

/* The gradient of ginex_combine: dz[slot, :] = weights[r * top + j] * dy[r, :], rows from offsets[experts]
 * on cleared, and dweights[r * top + j] = <dy[r, :], z[slot, :]> in f32, 0 for a pair without a slot. */
int32_t ginex_combine_backward(const ginex_routing_t* route /*host struct*/,
                               const ginex_rows_t* dy /*host struct*/, const ginex_rows_t* z /*host struct*/,
                               const float* weights, const ginex_rows_t* dz /*host struct*/,
                               float* dweights, void* stream);

/* Keeps x in 8 bits; with an activation also y = f(x) in the same pass (GINEX_ACT_NONE: y is NULL).
 * y may be x. */
int32_t ginex_compress(const ginex_rows_t* x /*host struct*/, int32_t activation,
                       const ginex_rows_t* y /*host struct or NULL*/,
                       const ginex_codes_t* kept /*host struct*/, void* stream);

/* The values that the codes stand for, rounded to the type of `out` (exact in f32 and bf16). */
int32_t ginex_restore(const ginex_codes_t* kept /*host struct*/, const ginex_rows_t* out /*host struct*/,
                      void* stream);

/* dx = dy * f'(x), x as the codes stand for it; relu: dy where x > 0, else 0.  NaN where x is.  dx may be dy. */
int32_t ginex_activate_backward(const ginex_codes_t* kept /*host struct*/, int32_t activation,
                                const ginex_rows_t* dy /*host struct*/,
                                const ginex_rows_t* dx /*host struct*/, void* stream);

/* Weight gradients of one linear layer per expert: with x the rows that the codes stand for,
 * dw[e, c, d] = sum over the slots s of expert e of x[source[s], c] * dy[s, d], products exact (an f32 dy
 * below 2^-110 counts without what it has below 2^-133), sums in f32 in an order that depends on the shapes
 * and offsets alone; 0 for an expert without rows.  dw is
 * [experts x kept->width x dy->width], contiguous, below 2^33 elements an expert.  dy has rows * top rows, of which those from
 * offsets[experts] on are not read.  route NULL: one layer, one expert, slot s holds row s. */
size_t ginex_weight_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width,
                                             int64_t out_width);

int32_t ginex_weight_gradient(const ginex_codes_t* kept /*host struct*/,
                              const ginex_routing_t* route /*host struct or NULL*/,
                              const ginex_rows_t* dy /*host struct*/, float* dw, void* ws,
                              size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GINEX_TRAIN_H */
