/*
 * sky_experts.h -- layers of experts beside a slice.
 *
 * In the place of a layer's feed-forward block a model may have several (experts), of
 * which every token takes a few: a router's logits choose them, the tokens' rows are
 * sorted by expert, every expert works on its own rows, and a token's results are added
 * up.  These are the steps of such a block, forward and backward, one by one:
 *   sky_route_*             logits -> experts, weights, and where every row goes
 *   sky_dispatch_*          tokens' rows -> the experts' order
 *   sky_grouped_gemm        the experts' linear maps and their gradients
 *   sky_grouped_column_sum  their bias gradients
 *   sky_combine_*           the weighted sum of a token's rows
 * The common rules of sky_ops.h hold (caller-owned device buffers, row-major matrices,
 * everything on `stream`).  A choice is a token's c-th expert; "rows" are the choices in
 * the experts' order, so there are up to tokens * top_k of them.
 */
#ifndef SKY_EXPERTS_H
#define SKY_EXPERTS_H

#include <stddef.h>
#include <stdint.h>

#include "sky_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Routing -----------------------------------------------------------------
 * A choice's weight is its probability under a softmax over all experts' logits, or
 * over those of the chosen ones alone (which then add up to 1). */
typedef enum { SKY_ROUTE_OVER_ALL = 0, SKY_ROUTE_OVER_CHOSEN = 1 } sky_route_weights;

typedef struct {
  int32_t tokens, experts, top_k;
  sky_dtype dtype;            /* of the logits and their gradients */
  sky_route_weights weights;
} sky_route_shape;

/* Scratch bytes of sky_route_fwd; 0 for a shape that it refuses.  The workspace must be
 * 4-byte aligned. */
size_t sky_route_workspace_bytes(const sky_route_shape* shape);

/* Chooses for every row of logits [tokens, experts] its top_k experts, largest logit
 * first, the lower index among equals, and writes
 *   expert: int32 [tokens, top_k], the chosen ones, -1 where there is none;
 *   weight: fp32 [tokens, top_k], 0 where there is none;
 *   row:    int32 [tokens, top_k], the choice's place when all choices are sorted by
 *           expert and, within one, by token (-1 where there is none);
 *   offset: int32 [experts + 1], where each expert's rows start; offset[experts] is how
 *           many rows there are in all.
 * A logit of -inf or NaN is never chosen and has no probability, so experts can be
 * closed to a token, and a padded token (none left) has no rows; NaN sets bit 2 of
 * *d_status.  Logits of +inf share the probability.  Deterministic.
 * Calls that may overlap on the GPU need a workspace each.
 * Errors: INVALID_ARG (null, sizes, top_k above experts, an unknown dtype or kind of
 * weights, a pointer off its type's grid, a workspace that is too small), UNSUPPORTED
 * (more than 1024 experts, top_k above 32, tokens * experts or tokens * top_k of 2^31 or more). */
sky_status sky_route_fwd(const sky_route_shape* shape, const void* logits, int32_t* expert,
                         float* weight, int32_t* row, int32_t* offset, void* workspace,
                         size_t workspace_bytes, int32_t* d_status, void* stream);

/* Its backward, from the forward's logits and experts and dweight = dL/dweight (fp32
 * [tokens, top_k]; what stands where there is no choice is not used): writes dlogits
 * [tokens, experts].  With p the softmax that the weights come from and
 * s = sum over the choices of p dweight: p (dweight - s) at the chosen experts; at the
 * others -p s (over all) or 0 (over the chosen).  dlogits may be logits.
 * Errors as the forward's. */
sky_status sky_route_bwd(const sky_route_shape* shape, const void* logits, const int32_t* expert,
                         const float* dweight, void* dlogits, void* stream);

/* ---- Rows to the experts and back ------------------------------------------------
 * tokens x width matrices (x, dx, y, dy) and tokens * top_k x width ones (rows, drows),
 * in dtype; row: int32 [tokens, top_k] as sky_route_fwd writes it.  Places outside
 * [0, tokens * top_k) are choices without a row: nothing is read or written for them.
 * Rows that no choice names are left as they are.  Sums are fp32, in the order of the
 * choices, and rounded once.  Outputs may not overlap inputs but where that is said.
 * Errors: INVALID_ARG (null, sizes, an unknown dtype, row, weight or dweight off the
 * 4-byte grid), UNSUPPORTED (width not a multiple of 16 bytes or above 2^20 values,
 * matrices not 16-byte aligned, top_k above 32, tokens * top_k of 2^31 or more). */
typedef struct {
  int32_t tokens, top_k, width;
  sky_dtype dtype;
} sky_rows_shape;

/* rows[row[t, c]] = x[t].  No place may be named twice. */
sky_status sky_dispatch_fwd(const sky_rows_shape* shape, const void* x, const int32_t* row,
                            void* rows, void* stream);
/* dx[t] = sum over c of drows[row[t, c]]; 0 for a token without rows. */
sky_status sky_dispatch_bwd(const sky_rows_shape* shape, const void* drows, const int32_t* row,
                            void* dx, void* stream);
/* y[t] = sum over c of weight[t, c] rows[row[t, c]]; 0 for a token without rows. */
sky_status sky_combine_fwd(const sky_rows_shape* shape, const void* rows, const int32_t* row,
                           const float* weight, void* y, void* stream);
/* drows[row[t, c]] = weight[t, c] dy[t] and dweight[t, c] = dot(dy[t], rows[row[t, c]])
 * (fp32 [tokens, top_k], 0 where there is no row).  No place may be named twice.  drows
 * may be rows. */
sky_status sky_combine_bwd(const sky_rows_shape* shape, const void* rows, const void* dy,
                           const int32_t* row, const float* weight, void* drows, float* dweight,
                           void* stream);

/* ---- Products grouped by expert ----------------------------------------------------
 * `groups` linear maps W_g [out, in], stored one after the other, each over its own rows
 * of a ragged matrix: group g has the rows [d_offset[g], d_offset[g + 1]) (int32
 * [groups + 1], never decreasing, within [0, rows], as sky_route_fwd writes it); `rows` is
 * how many the matrices hold.  Groups may be empty. */
typedef struct {
  int32_t groups, rows, out, in;
  sky_dtype dtype;
} sky_grouped_shape;

/* Scratch bytes of sky_grouped_gemm; 0 for a call that it refuses.  The workspace must be
 * 16-byte aligned.  (The present kernels write nothing to it.) */
size_t sky_grouped_gemm_workspace_bytes(sky_gemm_form form, const sky_grouped_shape* shape,
                                        sky_dtype out_dtype);

/* The contraction forms of sky_gemm for every group, with fp32 accumulation:
 *   XWT: C[r, out] = A[r, in] W_g^T   A [rows, in],  B the weights,  C [rows, out]
 *   XW : C[r, in]  = A[r, out] W_g    A [rows, out], B the weights,  C [rows, in]
 *   XTW: C_g = A_g^T B_g              A [rows, out], B [rows, in],   C fp32 [groups][out][in],
 *        zeros for a group without rows
 * Rows of C (and aux_out) that belong to no group are left as they are; rows of A and B
 * that belong to none may hold anything.
 * out_dtype: dtype for XWT and XW, FP32 for XTW.  Epilogues are sky_gemm's: STORE;
 * BIAS_GELU for XWT, aux_out [rows, out] being GELU' (fp16 for bf16, else fp32); GELU_BWD
 * for XW, times aux [rows, in].  bias: [groups][out] in dtype, or NULL, for XWT (BIAS_GELU
 * without one is GELU of the product).
 * C and aux_out may not overlap the operands.  Deterministic.  Calls that may overlap on
 * the GPU need a workspace each.
 * Errors: INVALID_ARG (null, sizes, an unknown dtype, form or epilogue, a pointer off its
 * type's grid, a workspace that is too small or not 16-byte aligned), UNSUPPORTED (other
 * output dtypes and epilogues; bf16: out or in not a multiple of 8, A, B, C, aux or aux_out
 * not 16-byte aligned; more than 1024 groups, 2^28 rows or more, out or in above 2^20,
 * groups * out of 2^31 or more, or 2^31 tiles of 64 x 64 or more); offsets that decrease or leave [0, rows] are clamped and
 * set bit 0 of *d_status, and what the calls then write is not defined within C. */
sky_status sky_grouped_gemm(sky_gemm_form form, const sky_grouped_shape* shape,
                            const int32_t* d_offset, const void* A, const void* B, void* C,
                            sky_dtype out_dtype, sky_epilogue epilogue, const void* bias,
                            const void* aux, void* aux_out, void* workspace,
                            size_t workspace_bytes, int32_t* d_status, void* stream);

/* out[g, n] = sum over the rows r of group g of x[r, n] (fp32, fixed order): the bias
 * gradients.  x: [rows, shape->out] in dtype; out: [groups, shape->out]; shape->in is not
 * used.  x and its width may be on any grid (16 bytes is faster).
 * Errors as sky_grouped_gemm's. */
sky_status sky_grouped_column_sum(const sky_grouped_shape* shape, const int32_t* d_offset,
                                  const void* x, float* out, int32_t* d_status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SKY_EXPERTS_H */
