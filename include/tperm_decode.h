/*
 * tperm, what answers with a mixture-of-experts layer need beside tperm_experts.h -- the router's choice and its
 * gradient, matrices held in 4 bits, products of few rows with them, and a whole layer for a few tokens
 * (AMD MI355X, gfx950).
 *
 * What tperm_experts.h says of all its calls holds here too: types, strides, alignment, streams, statuses, and that a
 * call allocates nothing, keeps nothing, does not wait, can be captured into a graph, and gives the same bits
 * for the same values however its work is scheduled.  Sums are formed in binary32.  Limits: 1 <= slots <= 64,
 * 1 <= experts <= 1024, tokens * slots < 2^31, rows < 2^31, widths (k, n, width, 2 * hidden) from 1 to 2^20, strides up to 2^28.
 */
#ifndef TPERM_DECODE_H
#define TPERM_DECODE_H

#include "tperm_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The router's choice.  expert[t, s], s = 0 .. slots-1: the experts with the largest scores of token t, largest first,
 * of equal scores the lowest expert first.  weights[t, s]: the softmax over those scores, or with over_all their part of the
 * softmax over all scores.  A score of minus infinity, or NaN, bars its expert: it is not chosen and counts as
 * exp(-inf) = 0.  Where fewer experts than slots are left, the remaining slots hold -1 and the weight 0, so a token all of
 * whose scores are barred goes nowhere.  Where scores are plus infinity, the softmax is its limit: those share
 * the weight equally.  scores: tokens rows of `experts` elements of `type`; expert and weights (binary32) are dense and what
 * the calls of tperm_experts.h take. */
tperm_status_t tperm_expert_route(const void *scores, int64_t scores_stride, int32_t *expert, float *weights,
                                  int64_t tokens, int64_t slots, int64_t experts, int over_all, int type, void *hip_stream);

/* The gradient of tperm_expert_route's weights brought back to all scores (the choice itself has none).  With
 * m = sum over s of weights[t, s] * grad_weights[t, s], over the slots that hold an expert,
 *   grad_scores[t, e] = sum over the slots s of e of weights[t, s] * (grad_weights[t, s] - m)      or with over_all
 *   grad_scores[t, e] = sum over the slots s of e of weights[t, s] * grad_weights[t, s]  -  p[t, e] * m,
 * p the softmax over all scores, which only this form reads (scores may be NULL without over_all; of the type of grad_scores).
 * Experts that are barred or not chosen have a gradient of zero, or of -p m.  expert and weights are those of the forward call;
 * an entry outside 0 .. experts-1 holds no expert, and its weight and gradient are not looked at. */
tperm_status_t tperm_expert_route_backward(const float *grad_weights, const void *scores, int64_t scores_stride,
                                           const int32_t *expert, const float *weights, void *grad_scores,
                                           int64_t grad_scores_stride, int64_t tokens, int64_t slots, int64_t experts,
                                           int over_all, int type, void *hip_stream);

/* Hold the rows of a matrix in 4 bits.  Every 32 neighbours of a row (a group; the last may be shorter) share a scale 2^s,
 * the least power of two with  max |x| <= 6 * 2^s,  -125 <= s <= 125; an element's code is x / 2^s rounded to nearest even in
 * the 4-bit type of 2 exponent bits and 1 mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6, and 8 more for their
 * negatives), held to 6 where s = 125 is too small.  A group with an infinity or NaN has the scale byte 255 and is NaN
 * as a whole.  codes: rows * TPERM_FOUR_BIT_GROUPS(width) * 16 bytes on 16 bytes, element i of a row in the low (even i) or high
 * half of byte i / 2, zeros behind its end; scales: rows * TPERM_FOUR_BIT_GROUPS(width) bytes, s + 127 each.
 * 17/32 bytes an element; the error of a value is at most 2^-2 of it, or 2^s / 4 where that is more. */
#define TPERM_FOUR_BIT_GROUPS(width) (((width) + 31) / 32)
tperm_status_t tperm_four_bit_store(const void *x, int64_t x_stride, uint8_t *codes, uint8_t *scales, int64_t rows,
                                    int64_t width, int type, void *hip_stream);

/* The values that codes and scales stand for, rounded to `type` and held to its finite range (exact in binary32
 * and bfloat16).  Scales of 2 .. 252 are powers of two as above, 255 is NaN; other bytes are not made by
 * tperm_four_bit_store and stand for no particular value. */
tperm_status_t tperm_four_bit_load(const uint8_t *codes, const uint8_t *scales, void *out, int64_t out_stride,
                                   int64_t rows, int64_t width, int type, void *hip_stream);

/* Products with a matrix held in 4 bits:  out[r, j] = sum over i of x[r, i] * w[j, i],  w the n rows of k elements that
 * codes and scales stand for.  Values are multiplied as they stand, neither they nor x are rounded first (of binary32 numbers below
 * 2^-102 not all bits may count).  Made for few rows, when
 * the matrix is what there is to read: it is read once for every 64 of them.  Any number of rows is right.
 * TOO_LARGE: codes of more than 2^32 - 256 bytes. */
tperm_status_t tperm_four_bit_product(const void *x, int64_t x_stride, const uint8_t *codes, const uint8_t *scales,
                                      void *out, int64_t out_stride, int64_t rows, int64_t k, int64_t n, int type,
                                      void *hip_stream);

/* A whole layer for a few tokens:
 *   out[t] = sum over s of weights[t, s] * w_out[e] (g * sigmoid(g) * u),   (g, u) = the halves of w_in[e] x[t],   e = expert[t, s]
 * over the slots whose number is in 0 .. experts-1 (zeros where a token has none; the weights of the others are not looked
 * at).  x, out: tokens rows of width elements, tokens <= TPERM_FEW_TOKENS; w_in: experts matrices of 2 * hidden rows of width
 * elements; w_out: of width rows of hidden elements, dense.  w_in_scales and w_out_scales both NULL: the matrices are of `type`.
 * Both given: w_in and w_out are the codes of tperm_four_bit_store of all rows of all experts.  weights NULL: ones.
 * What lies between the two products, weights * g * sigmoid(g) * u, is held in binary32 whatever `type` is, with its bits and its range (beside matrices of
 * bfloat16 or 4 bits not all bits of numbers below 2^-102 may count).  Every expert that is
 * named is read once for every 32 tokens that name it, others not at all.  A token that names an expert twice gives it the sum of both weights.
 * workspace: tperm_expert_few_workspace(...) bytes on 16 bytes, apart from the other arrays; overwritten; two calls that use
 * the same one at the same time race.  TOO_LARGE: too small a workspace, or one expert's matrix (its codes) of more than 2^32 - 256
 * bytes. */
#define TPERM_FEW_TOKENS 64
size_t tperm_expert_few_workspace(int64_t tokens, int64_t slots, int64_t experts, int64_t width, int64_t hidden, int type,
                                  int four_bits);
tperm_status_t tperm_expert_few(const void *x, int64_t x_stride, const int32_t *expert, const float *weights,
                                const void *w_in, const uint8_t *w_in_scales, const void *w_out, const uint8_t *w_out_scales,
                                void *out, int64_t out_stride, void *workspace, size_t workspace_bytes, int64_t tokens,
                                int64_t slots, int64_t experts, int64_t width, int64_t hidden, int type, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TPERM_DECODE_H */
