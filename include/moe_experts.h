/*
 * moe_experts.h - C ABI of the operators around and inside the experts that
 * a program calls one by one on MI355X: the sort of a router's choice by
 * expert, the rows' way to the experts and back with its gradients, and the
 * experts' products in microscaled 4-bit floating point.  Same library,
 * status codes and conventions as moe_gemm2.h: extern "C", nothing throws,
 * aborts or prints, the caller owns every buffer, calls only enqueue on
 * "stream", tensors are dense and row-major.
 *
 * What they compute, with S = T topk slots s = (t, j):
 *
 *   sort      a slot is kept iff first <= expert_ids[s] < first + E; rows are
 *             the kept slots by expert, then by slot (a stable sort):
 *             row(s) = offsets[e(s)] + #{kept s' < s of the same expert}
 *   dispatch  out[row(t, j), :] = x[t, :]
 *             and its gradient   dx[t, :] = sum_j d[row(t, j), :]
 *   combine   out[t, :] = sum_j gates[t, j] y[row(t, j), :]
 *             and its gradient   dy[row(t, j), :] = gates[t, j] dout[t, :],
 *                                dgates[t, j] = sum_c y[row(t, j), c] dout[t, c]
 *   product   out[r, n] = sum_k a[id(r), k] w[e(r), n, k] of operands in
 *             microscaled 4-bit floating point (mx4 below)
 *
 * "slot_rows" [T, topk] int32 holds row(s), or -1 for a slot without a row.
 * Slots without a row add nothing (not 0 times something), get no row and
 * have dgates = 0.  A slot_rows entry below -1 or at or past `rows` is taken
 * as -1 and flagged: where `workspace` (a moe_gemm2 workspace of at least
 * 512 bytes, of which only the status word is used) is not NULL,
 * moe_gemm2_status reports MOE_ERR_BAD_ROUTING.  Rows that no slot has are
 * not written; what a row that several slots have then holds is not defined (each
 * of them writes it).  Outputs overlap neither inputs nor each other, except that
 * combine's dy may be its y; the same address for an input of rows and the output
 * is MOE_ERR_INVALID_ARG.
 * T, rows >= 0, 1 <= topk <= 64, 1 <= H < 2^31 - 4096 (elements; dispatch: bytes
 * of a row below 2^31), rows < 2^31, else MOE_ERR_INVALID_ARG or, past an upper
 * limit, MOE_ERR_UNSUPPORTED.
 * Sums over slots are taken in fp32 in slot order and rounded once (round to
 * nearest even) to the output's type, so results do not vary from run to
 * run.
 *
 * mx4: blocks of 32 consecutive elements along K, KB = ceil(K / 32) of them
 * per row, the last one filled up with zeros.  A block's scale is
 * 2^X, X = max(floor(log2(max |x|)) - 2, -127), held as the byte X + 127; its
 * elements are x / 2^X rounded to the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}
 * (ties to the even code, larger values to 6), held as sign and index in 4
 * bits.  All zeros: X = -127.  A block that holds an infinity or a NaN has
 * scale byte 255 and codes 0: all of it is NaN.  (This is the MXFP4 format of
 * the OCP Microscaling specification, version 1.0.)
 *   codes   uint8 [rows, 16 KB]: element 2i in the low, 2i + 1 in the high
 *           half of byte i of its row (16-byte aligned)
 *   scales  uint8 [rows, KS], KS = 4 ceil(KB / 4): a block's byte each, then
 *           zeros (4-byte aligned)
 */
#ifndef MOE_EXPERTS_H
#define MOE_EXPERTS_H

#include "moe_gemm2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MOE_BF16 = 0, MOE_F32 = 1 } moe_type_t;

/* ---- tokens sorted by expert ------------------------------------------- */

/* Bytes of scratch moe_sort_by_expert needs (0 for up to 4096 slots and for
 * invalid arguments); its contents do not matter, before or after. */
size_t moe_sort_scratch_size(int32_t T, int32_t topk, int32_t E);

/* The sort, in one launch for up to 4096 slots and two beyond.
 *   expert_ids      device int32 [T, topk]: ids outside [first, first + E) are
 *                   slots without a row (dropped, or another GPU's expert); a
 *                   token may name an expert twice
 *   gates           device fp32 [T, topk]
 *   expert_offsets  device int32 [E + 1]
 *   token_ids       device int32 [T topk]: the token of each row, then -1
 *   gate_w          device fp32 [T topk]: the gate of each row, then 0
 *   slot_rows       device int32 [T, topk]
 * expert_offsets, token_ids and gate_w are what moe_gemm2_combine,
 * moe_gemm1_swiglu and moe_layer_forward take with rows = T topk.
 * T >= 0, 1 <= topk <= 64, 1 <= E <= 1024, T topk < 2^31 - 2^24 (else
 * MOE_ERR_INVALID_ARG or, past a limit, MOE_ERR_UNSUPPORTED). */
int moe_sort_by_expert(const int32_t* expert_ids, const float* gates, int32_t* expert_offsets,
                       int32_t* token_ids, float* gate_w, int32_t* slot_rows, int32_t T,
                       int32_t topk, int32_t E, int32_t first_expert, void* scratch,
                       size_t scratch_bytes, void* stream);

/* ---- rows to the experts and back --------------------------------------- */

/* x [T, row_bytes] to out [rows, row_bytes]; the type does not matter. */
int moe_dispatch_rows(const void* x, const int32_t* slot_rows, void* out, int32_t T, int32_t topk,
                      int64_t rows, int64_t row_bytes, void* workspace, void* stream);

/* d [rows, H] of d_type to dx [T, H] of dx_type (MOE_BF16 or MOE_F32, aligned
 * to their elements), fully written. */
int moe_dispatch_rows_grad(const void* d, const int32_t* slot_rows, void* dx, int32_t T,
                           int32_t topk, int64_t rows, int32_t H, int32_t d_type, int32_t dx_type,
                           void* workspace, void* stream);

/* y [rows, H] of y_type, gates fp32 [T, topk], to out [T, H] of out_type, fully
 * written. */
int moe_combine_rows(const void* y, const int32_t* slot_rows, const float* gates, void* out,
                     int32_t T, int32_t topk, int64_t rows, int32_t H, int32_t y_type,
                     int32_t out_type, void* workspace, void* stream);

/* dout [T, H] of dout_type and y [rows, H] of y_type to dy [rows, H] of y_type
 * and dgates fp32 [T, topk] (fully written). */
int moe_combine_rows_grad(const void* dout, const void* y, const int32_t* slot_rows,
                          const float* gates, void* dy, float* dgates, int32_t T, int32_t topk,
                          int64_t rows, int32_t H, int32_t dout_type, int32_t y_type,
                          void* workspace, void* stream);

/* ---- microscaled 4-bit floating point ----------------------------------------- */

/* x [rows, K] of x_type (aligned to its elements) to codes and scales (format
 * above), every byte of which is written.  rows >= 0, 1 <= K < 2^31 - 256, and rows
 * times K (rounded up to 32) below 2^35, else MOE_ERR_INVALID_ARG or, past an upper
 * limit, MOE_ERR_UNSUPPORTED. */
int moe_mx4_quantize(const void* x, void* codes, void* scales, int64_t rows, int32_t K,
                     int32_t x_type, void* stream);

/* Weights as the rest of the library takes them, w [E, K, N] of w_type, to codes
 * [E, N, 16 KB] and scales [E, N, KS] for moe_mx4_product: blocks along K, rows
 * along N.  Done once, as the weights are loaded.  K and N below 2^31 - 256, E times K
 * (rounded up to 256) times N (to 128) below 2^39. */
int moe_mx4_quantize_weights(const void* w, void* codes, void* scales, int32_t E, int32_t K,
                             int32_t N, int32_t w_type, void* stream);

/* The values that codes and scales stand for, to out [rows, K] of out_type
 * (exact in both types).  Limits as for moe_mx4_quantize. */
int moe_mx4_dequantize(const void* codes, const void* scales, void* out, int64_t rows, int32_t K,
                       int32_t out_type, void* stream);

/* The experts' products.
 *   a_codes, a_scales  device, a [a_rows, K] in mx4
 *   w_codes, w_scales  device, w [E, N, K] in mx4
 *   expert_offsets     device int32 [E + 1], as for moe_gemm2_combine
 *   row_ids            device int32 [rows]: the row of a that each row takes (the
 *                      dispatch gather: token_ids); NULL: row r takes a's row r.
 *                      A row outside [0, a_rows) counts as zeros and is flagged as
 *                      slot_rows entries are (with NULL: is zeros)
 *   out                device bf16 [rows, N], or with swiglu != 0 (N even) [rows,
 *                      N / 2]: silu(p[:, n]) * p[:, N / 2 + n] of the product p; rows
 *                      from expert_offsets[E] on are not written
 * Products are exact, sums are fp32, the activation is fp32, out is rounded
 * once (to nearest even).  A NaN block makes the sums it enters NaN.  Pad
 * bytes of scales are not used.  1 <= E <= 1024; a_rows >= 1 where rows > 0; rows and K below
 * 2^31 - 256; the codes of a, and of one expert's weights, below 2 GiB each (else
 * MOE_ERR_UNSUPPORTED). */
int moe_mx4_product(const void* a_codes, const void* a_scales, const void* w_codes,
                    const void* w_scales, const int32_t* expert_offsets, const int32_t* row_ids,
                    void* out, int64_t a_rows, int64_t rows, int32_t K, int32_t N, int32_t E,
                    int32_t swiglu, void* workspace, void* stream);

/* Bytes of scratch moe_mx4_layer_forward needs (0 for invalid arguments); its
 * contents do not matter, before or after. */
size_t moe_mx4_layer_scratch_size(int32_t T, int32_t H, int32_t I, int32_t topk);

/* The post-router layer with its experts in 4 bits: hidden quantised; the
 * up-projection with the token gather and SwiGLU; its outputs, rounded to bf16,
 * quantised (by the up-projection itself in long calls, by a launch in short ones);
 * the down-projection (bf16); the combine.  Four or five launches on stream, and the
 * result is that of the separate calls bit for bit.
 *   hidden          device bf16 [T, H]
 *   w1              mx4 [E, 2 I, H]: an expert's I gate rows, then its I up rows
 *   w2              mx4 [E, H, I]
 *   expert_offsets, token_ids, slot_rows
 *                   as moe_sort_by_expert writes them (token_ids [T topk])
 *   gates           device fp32 [T, topk]
 *   out             device [T, H] of out_type, fully written
 *   scratch         16-byte aligned, moe_mx4_layer_scratch_size bytes
 *   workspace       NULL, or where bad entries are flagged
 * Limits as for the functions it runs. */
int moe_mx4_layer_forward(const void* hidden, const void* w1_codes, const void* w1_scales,
                          const void* w2_codes, const void* w2_scales,
                          const int32_t* expert_offsets, const int32_t* token_ids,
                          const int32_t* slot_rows, const float* gates, void* out, int32_t T,
                          int32_t H, int32_t I, int32_t E, int32_t topk, int32_t out_type,
                          void* scratch, size_t scratch_bytes, void* workspace, void* stream);

/* ABI version of this header (major * 100 + minor): 100. */
int moe_experts_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MOE_EXPERTS_H */
