/*
 * tperm, mixture-of-experts operators -- permutations of rows that are known only on the GPU, the
 * products between them, and activations kept in 8 bits for the backward pass (AMD MI355X, gfx950).
 *
 * A layer has `experts` matrices.  Every one of `tokens` tokens names `slots` of them; assignment
 * a = t * slots + s is slot s of token t.  tperm_expert_sort brings the assignments into the order of
 * their experts:
 *
 *   source[r]   the assignment at row r of the sorted order (a permutation of 0 .. rows-1, rows =
 *               tokens * slots; within an expert assignments keep their order)
 *   place[a]    its inverse
 *   offsets[e]  first row of expert e, e = 0 .. experts; rows from offsets[experts] on are those of
 *               assignments that name no expert, and are called unused below
 *
 * All other calls take these maps, so a program that makes its own order can use them too.  Maps are read
 * on the GPU and not checked on the host: offsets have to rise from 0 to at most `rows`, source and place
 * have to be permutations of 0 .. rows-1.  An entry of source or place outside that range is treated as
 * unused, by the products as a row of zeros; nothing is read or written outside the tensors for it.
 *
 * Element types are a tperm_type_t.  Sums, products of the gates and scales are formed in binary32 and
 * rounded once, to nearest even, where they are stored.  A matrix of rows is given by a pointer to its first
 * element and a stride in elements between rows (>= its width); elements of a row are neighbours.  Any
 * alignment to the element's size is right; rows that start on 16 bytes (pointer and stride) are read and
 * written fastest.  Expert matrices, maps, weights, codes and scales are dense.
 *
 * All calls enqueue kernels on hip_stream and return; no device memory is allocated, nothing is kept from
 * one call to the next, and no call synchronises, copies or clears memory through the runtime, so all may be
 * captured into a graph.  Pointers are DEVICE pointers owned by the caller.  Results do not depend on
 * how the work is scheduled: the same call on the same values gives the same bits.
 *
 * Limits: rows < 2^31, 1 <= slots <= 64, 1 <= experts <= 1024, widths (k, n, width) from 1 to 2^20,
 * strides up to 2^28.
 * Statuses: NULL (a pointer that is needed; arrays of no elements are not looked at), DIMS (a size or stride
 * outside its limits), ELEM_SIZE (a type that the call does not know), TOO_LARGE (rows >= 2^31, a workspace
 * that is too small, an operand of a product beyond the size stated there), ALIGN (a pointer that is no
 * multiple of its element's size), ALIAS (an output overlaps another tensor of the call, from first
 * to last byte), HIP.  The checks come before any launch.
 */
#ifndef TPERM_EXPERTS_H
#define TPERM_EXPERTS_H

#include "tperm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TPERM_TYPE_F32 = 0,  /* IEEE binary32 */
    TPERM_TYPE_F16 = 1,  /* IEEE binary16 */
    TPERM_TYPE_BF16 = 2  /* bfloat16      */
} tperm_type_t;

#define TPERM_EXPERTS_MAX 1024
#define TPERM_SLOTS_MAX 64
#define TPERM_WIDTH_MAX (1 << 20)

/* Order the assignments by expert.  expert: tokens * slots numbers; any number outside 0 .. experts-1 names no
 * expert.  offsets: experts + 1 numbers, source and place: tokens * slots, all overwritten.  workspace:
 * TPERM_EXPERT_SORT_WORKSPACE_BYTES(tokens * slots, experts) bytes, 4-byte aligned, apart from the other
 * arrays; its contents are overwritten; two calls that use the same one at the same time race.  It is not
 * looked at for up to TPERM_EXPERT_SORT_ONE_BLOCK assignments. */
#define TPERM_EXPERT_SORT_ONE_BLOCK 8192
#define TPERM_EXPERT_SORT_WORKSPACE_BYTES(rows, experts) \
    ((rows) <= TPERM_EXPERT_SORT_ONE_BLOCK ? (size_t)0 : (size_t)128 * ((size_t)(experts) + 1) * 4)
tperm_status_t tperm_expert_sort(const int32_t *expert, int64_t tokens, int64_t slots, int64_t experts,
                                 int32_t *offsets, int32_t *source, int32_t *place, void *workspace,
                                 size_t workspace_bytes, void *hip_stream);

/* Rows to their experts:  out[r] = weights[source[r]] * x[source[r] / slots]  for the used rows, zeros for
 * the others.  x: tokens rows of `width` elements; out: tokens * slots rows; weights: tokens * slots binary32
 * numbers, or NULL for ones.  With weights it is the gradient of tperm_expert_combine to its rows. */
tperm_status_t tperm_expert_gather(const void *x, int64_t x_stride, const int32_t *source, const int32_t *offsets,
                                   const float *weights, void *out, int64_t out_stride, int64_t tokens, int64_t slots,
                                   int64_t experts, int64_t width, int type, void *hip_stream);

/* Results back to their tokens:  out[t] = sum over s of weights[t, s] * rows[place[t, s]], over the used rows
 * (zeros where a token has none; unused rows are not read).  The sum runs over s in order, in binary32.
 * weights NULL: ones, which is the gradient of tperm_expert_gather without weights. */
tperm_status_t tperm_expert_combine(const void *rows, int64_t rows_stride, const int32_t *place, const int32_t *offsets,
                                    const float *weights, void *out, int64_t out_stride, int64_t tokens, int64_t slots,
                                    int64_t experts, int64_t width, int type, void *hip_stream);

/* Gradients of tperm_expert_combine from grad, that of its result (tokens rows):
 *   grad_rows[place[t, s]] = weights[t, s] * grad[t]       (zeros for unused rows)
 *   grad_weights[t, s]     = sum over c of grad[t, c] * rows[place[t, s], c]       (0 for unused rows)
 * in one pass over grad and rows.  weights and grad_weights are binary32. */
tperm_status_t tperm_expert_combine_backward(const void *grad, int64_t grad_stride, const void *rows, int64_t rows_stride,
                                             const int32_t *place, const int32_t *offsets, const float *weights,
                                             void *grad_rows, int64_t grad_rows_stride, float *grad_weights,
                                             int64_t tokens, int64_t slots, int64_t experts, int64_t width, int type,
                                             void *hip_stream);

/* The experts' products:  out[r, j] = sum over i of x[row(r), i] * w[e(r)](i, j),  e(r) the expert of row r,
 * for the used rows; zeros for the others.  source NULL: row(r) = r; else row(r) = source[r] / slots, so that
 * rows need not be gathered first.  x: x_rows rows of k elements; out: `rows` rows of n elements; w: experts
 * matrices of one type with x and out, w(i, j) at j + n * i, or with w_k_first at i + k * j (the summed index
 * first, the layout of a linear layer's weight).  The gradient to the rows is the same call with k and n
 * changed for each other, the same w and the other w_k_first.
 * TOO_LARGE: with source, x of more than 2^32 - 256 bytes; one expert's matrix of more than that. */
tperm_status_t tperm_expert_product(const void *x, int64_t x_stride, int64_t x_rows, const int32_t *source, int64_t slots,
                                    const int32_t *offsets, const void *w, int w_k_first, void *out, int64_t out_stride,
                                    int64_t rows, int64_t experts, int64_t k, int64_t n, int type, void *hip_stream);

/* Gradient to the experts' matrices:  out[e](i, j) = sum over the rows r of expert e of
 * x[row(r), i] * grad[r, j],  zeros for an expert without rows; with accumulate it is added to what out holds.
 * Layout of out and row(r) as in tperm_expert_product; out_type is the element type of out.
 * x_scales NULL: x is of `type`; else x points to the codes and x_scales to the scales of a
 * tperm_checkpoint_store of x_rows rows of width k (x_stride is not looked at), and the values that they stand
 * for, rounded to `type` and held to its finite range, are multiplied.
 * TOO_LARGE: as above, the matrix being of out_type and x in the form it has; grad may be of any size. */
tperm_status_t tperm_expert_weight_gradient(const void *x, int64_t x_stride, const uint8_t *x_scales, int64_t x_rows,
                                            const int32_t *source, int64_t slots, const void *grad, int64_t grad_stride,
                                            const int32_t *offsets, void *out, int out_type, int w_k_first, int accumulate,
                                            int64_t rows, int64_t experts, int64_t k, int64_t n, int type,
                                            void *hip_stream);

/* Keep rows in 8 bits.  Every 32 neighbours of a row (the last block may be shorter) share a scale 2^s, the
 * least power of two with  max |x| <= 448 * 2^s  over the block's finite values, -117 <= s <= 120; a
 * value's code is x / 2^s rounded to nearest even in the 8-bit type of 4 exponent and 3 mantissa bits that has
 * no infinities (largest 448).  Infinities and NaN become NaN and do not touch their neighbours.  codes:
 * rows * width bytes; scales: rows * TPERM_CHECKPOINT_BLOCKS(width) bytes, s + 127 each.
 * 33/32 bytes an element; the error of a value is at most 2^-4 of it, or 2^-10 * 2^s where that is more. */
#define TPERM_CHECKPOINT_BLOCKS(width) (((width) + 31) / 32)
tperm_status_t tperm_checkpoint_store(const void *x, int64_t x_stride, uint8_t *codes, uint8_t *scales, int64_t rows,
                                      int64_t width, int type, void *hip_stream);

/* The values that codes and scales stand for, rounded to `type` and held to its finite range (they are exact
 * in binary32 below 2^128, and in bfloat16 unless smaller than its normal numbers).  Scales of 1 .. 254 are powers of two as
 * above. */
tperm_status_t tperm_checkpoint_load(const uint8_t *codes, const uint8_t *scales, void *out, int64_t out_stride,
                                     int64_t rows, int64_t width, int type, void *hip_stream);

/* The gated activation of rows [g, u] (g the first `width` elements, u the next):
 *   out = g * sigmoid(g) * u
 * and the same rows in 8 bits: codes rows * 2 * width bytes, scales rows * 2 * TPERM_CHECKPOINT_BLOCKS(width),
 * g's first, as two checkpoints beside each other.  codes and scales may both be NULL: nothing is kept.
 * In front of its rounding a result is within 9 * 2^-23 of its value, 16-bit ones within (9 + |g| / 2) * 2^-23, down to the
 * smallest numbers of the type: a sigmoid that is no normal number does not become zero. */
tperm_status_t tperm_gated_forward(const void *gates, int64_t gates_stride, void *out, int64_t out_stride, uint8_t *codes,
                                   uint8_t *scales, int64_t rows, int64_t width, int type, void *hip_stream);

/* Its backward pass from the codes and scales that tperm_gated_forward kept, in one pass, p = sigmoid(g):
 *   grad_gates = [grad * u * p * (1 + g * (1 - p)), grad * g * p]     out = g * p * u
 * out, the result again (the next product's weight gradient needs it), may be NULL. */
tperm_status_t tperm_gated_backward(const void *grad, int64_t grad_stride, const uint8_t *codes, const uint8_t *scales,
                                    void *grad_gates, int64_t grad_gates_stride, void *out, int64_t out_stride,
                                    int64_t rows, int64_t width, int type, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TPERM_EXPERTS_H */
