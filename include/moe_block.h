/*
 * moe_block.h - C ABI of what stands around the experts of a transformer block
 * on MI355X, from the residual stream to the residual stream: the router's
 * choice, the join of a block's output onto the stream with the norms on both
 * sides, and the post-router layer for a few tokens.  Same library, status codes
 * and conventions as moe_gemm2.h and moe_experts.h: extern "C", nothing throws,
 * aborts or prints, the caller owns every buffer, calls only enqueue on "stream",
 * which belongs to the current device, tensors are dense, row-major and aligned to
 * their elements where nothing else is said.  Types are moe_type_t.
 *
 * What they compute, for token t, expert e, slot j, column c:
 *
 *   choose  key[t, e] = logits[t, e] + bias[e] (in fp32); the topk largest keys of a
 *           token in falling order, equal keys in the order of e.  A key of -inf
 *           (an expert that the token may not take) or NaN is never chosen; slots
 *           without an expert have id -1 and gate 0.
 *           p[t, e] = exp(l[t, e]) / sum over all e of exp(l)     (softmax)
 *                     1 / (1 + exp(-l[t, e]))                     (sigmoid)
 *           gates[t, j] = scale p_j, or renormalised scale p_j / sum over the
 *           chosen of p.
 *   join    b = y, or with `after`  y rsqrt(mean_c(y^2) + eps) after[c]
 *           a = b, or with a gate   gate[t] b  or  gate[c] b
 *           x = h + scale drop(a), rounded to h's type
 *           z = x rsqrt(mean_c(x^2) + eps) before[c], of x as rounded
 *           drop(a) is a / (1 - p) or 0: the 32 random bits of element (t, c) are word
 *           c mod 4 of Philox4x32-10 (Salmon et al., "Parallel random numbers: as
 *           easy as 1, 2, 3", 2011) with the 64-bit key rng[0] and the counter
 *           (c / 4, t, low and high half of rng[1]); it is kept where they are at
 *           least floor(p 2^32).  The gradient makes the same bits again.
 *   few     out[t, :] = sum over experts e of
 *             G[t, e] (silu(x_t Wg_e) * (x_t Wu_e)) W2_e,
 *           G[t, e] the sum of the gates of t's slots that name e; experts that no
 *           slot of a token names add nothing to it (not 0 times something).
 *
 * Sums and statistics are fp32, in an order that sizes alone decide: results do not
 * vary from run to run.  Calls that may run at the same time (on two streams, or in two
 * graphs) need scratch of their own.
 */
#ifndef MOE_BLOCK_H
#define MOE_BLOCK_H

#include "moe_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the router's choice ------------------------------------------------ */

typedef enum { MOE_SOFTMAX = 0, MOE_SIGMOID = 1 } moe_score_t;

/* logits [T, E] of logits_type and bias fp32 [E] (or NULL) to ids int32 and gates
 * fp32 [T, topk].  T >= 0, 1 <= E <= 1024, 1 <= topk <= min(64, E). */
int moe_choose(const void* logits, const float* bias, int32_t* ids, float* gates, int32_t T,
               int32_t E, int32_t topk, int32_t logits_type, int32_t score, int32_t renormalize,
               float scale, void* stream);

/* dgates fp32 [T, topk], logits and the chosen ids to dlogits [T, E] of the logits'
 * type, fully written (the choice itself and the bias have no gradient).  A slot with
 * id -1 adds nothing; an id twice counts as two slots.  Other ids outside [0, E) are
 * taken as -1 and flagged in `workspace` (NULL, or as in moe_experts.h). */
int moe_choose_grad(const float* dgates, const void* logits, const int32_t* ids, void* dlogits,
                    int32_t T, int32_t E, int32_t topk, int32_t logits_type, int32_t score,
                    int32_t renormalize, float scale, void* workspace, void* stream);

/* ---- the residual join and its norms --------------------------------------- */

typedef enum { MOE_GATE_NONE = 0, MOE_GATE_TOKEN = 1, MOE_GATE_CHANNEL = 2 } moe_gate_t;

/* x and z as above.
 *   h        [T, H] of h_type, or NULL: nothing to add to (x = scale drop(a))
 *   y        [T, H] of y_type, or NULL: x is h and is not written
 *   after, before   [H] of w_type, or NULL: no such norm (before: z not written)
 *   gate     [T] or [H] of w_type, by gate_kind
 *   drop     p in [0, 1); 0: rng is not read
 *   rng      device uint64 [2], 8-byte aligned: seed and offset.  The call reads
 *            them as it runs, so a captured graph draws other numbers on every
 *            replay if the program changes them in between
 *   x        [T, H] of h_type; may be h
 *   z        [T, H] of z_type
 * Apart from x = h outputs overlap neither inputs nor each other; the same address
 * is MOE_ERR_INVALID_ARG.  T >= 0, 1 <= H <= 16384 (else MOE_ERR_UNSUPPORTED). */
int moe_join(const void* h, const void* y, const void* after, const void* gate, const void* before,
             const uint64_t* rng, void* x, void* z, int32_t T, int32_t H, int32_t h_type,
             int32_t y_type, int32_t z_type, int32_t w_type, int32_t gate_kind, float scale,
             double drop, float eps, void* stream);

/* Bytes of scratch moe_join_grad needs (0 for invalid arguments); its contents do not
 * matter, before or after. */
size_t moe_join_grad_scratch_size(int32_t T, int32_t H);

/* The gradients, from those of x and of z (either may be NULL: zeros):
 *   dx       [T, H] of h_type
 *   dz       [T, H] of z_type (with before)
 *   x        [T, H] of h_type as moe_join wrote it (without y: h); read with dz only
 *   y        [T, H] of y_type, or NULL as in the join; read with after or a gate only,
 *            and may be NULL without them also where the join had one
 *   dh       [T, H] of h_type, may be dx; NULL: not written
 *   dy       [T, H] of y_type (where the join had y); NULL: not written
 *   d_after, d_before   fp32 [H]; NULL: not written
 *   d_gate   fp32 [T] or [H]; NULL: not written
 * Apart from dh = dx outputs overlap neither inputs nor each other.  The columns'
 * sums (d_after, d_before, d_gate of channels) are fully written also for T = 0. */
int moe_join_grad(const void* dx, const void* dz, const void* x, const void* y, const void* after,
                  const void* gate, const void* before, const uint64_t* rng, void* dh, void* dy,
                  float* d_after, float* d_gate, float* d_before, int32_t T, int32_t H,
                  int32_t h_type, int32_t y_type, int32_t z_type, int32_t w_type,
                  int32_t gate_kind, float scale, double drop, float eps, void* scratch,
                  size_t scratch_bytes, void* stream);

/* ---- the post-router layer for a few tokens ---------------------------------- */

#define MOE_FEW_TOKENS 16

/* Bytes of scratch the calls below need (0 for invalid arguments); its contents do
 * not matter, before or after. */
size_t moe_few_scratch_size(int32_t T, int32_t H, int32_t I, int32_t E, int32_t topk);

/* The layer in two launches, without a sort, each hit expert's weights read once (in mx4, of
 * more than eight tokens, w1 once for every seven that name the expert).
 *   hidden      device bf16 [T, H] (16-byte aligned)
 *   w1, w2      as moe_layer_forward takes them: [E, H, 2 I] packed by
 *               moe_gemm1_pack_weights and [E, I, H], 16-byte aligned
 *   ids, gates  device int32 and fp32 [T, topk]: as moe_sort_by_expert takes
 *               them; ids outside [first, first + E) are slots without an expert
 *   out         device [T, H] of out_type, fully written
 *   scratch     16-byte aligned, moe_few_scratch_size bytes
 * 0 <= T <= MOE_FEW_TOKENS, 1 <= topk <= 64, 1 <= E <= 1024, H % 8 == 0, I % 16 == 0,
 * H, I <= 2^22, 4 H I < 2^31, min(T topk, E) I < 2^26 (else MOE_ERR_INVALID_ARG or
 * MOE_ERR_UNSUPPORTED).  Products in bf16, sums, activation and the weighted sum over experts in fp32; the activation goes into the
 * second product as two bf16 parts (16 bits of mantissa; one beyond bf16's range counts as
 * infinite), out is rounded once to its type.  An infinite weight of w2 makes NaN of the
 * sums that it enters, whichever sign they would have. */
int moe_few_forward(const void* hidden, const void* w1, const void* w2, const int32_t* ids,
                    const float* gates, void* out, int32_t T, int32_t H, int32_t I, int32_t E,
                    int32_t topk, int32_t first_expert, int32_t out_type, void* scratch,
                    size_t scratch_bytes, void* stream);

/* The same with weights in mx4 (w1 [E, 2 I, H]: an expert's I gate rows, then its I up
 * rows; w2 [E, H, I]) and activations in bf16: what a weight stands for is exact in the
 * products.  Limits as above, but any H and I whose codes are below 2 GiB an expert.  A
 * value below 2^-126 may count as zero.  NaN blocks make the sums that they enter NaN; pad
 * bytes of scales are not used. */
int moe_few_forward_mx4(const void* hidden, const void* w1_codes, const void* w1_scales,
                        const void* w2_codes, const void* w2_scales, const int32_t* ids,
                        const float* gates, void* out, int32_t T, int32_t H, int32_t I, int32_t E,
                        int32_t topk, int32_t first_expert, int32_t out_type, void* scratch,
                        size_t scratch_bytes, void* stream);

/* ABI version of this header (major * 100 + minor): 100. */
int moe_block_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MOE_BLOCK_H */
