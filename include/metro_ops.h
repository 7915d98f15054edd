/*
 * metro_ops.h -- single operators on caller-owned device buffers: the kernels
 * of libmetro.so's forward pass, exported so that each can be checked on its
 * own against a CPU reference (the model entry points in metro.h are what a
 * serving loop calls; these run one step of it), and the feed-forward block in
 * 8 bits, which that forward pass (bf16 throughout) does not use: it is for
 * callers that run layers of their own.
 *
 * All pointers are device pointers on the current HIP device; work is
 * enqueued on `stream` (a hipStream_t, NULL = default stream).  Return value
 * and metro_last_error() as in metro.h; a launch failure returns METRO_E_HIP.
 */
#ifndef METRO_OPS_H
#define METRO_OPS_H

#include <stdint.h>

#include "metro.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Weight layout of the projection GEMMs.  W_packed receives the bf16 matrix
 * W [N, Kp] (W[n, k] = W_rowmajor[n * ld + k] for k < K, 0 for K <= k < Kp) in
 * matrix-core operand order: 16 x 32 tiles (16 rows, 32 columns), tiles
 * row-major over (n / 16, k / 32), tile (tn, tk) stored as 64 chunks of 8
 * elements in the order c = r + 16 g, chunk c = W[16 tn + r][32 tk + 8 g ..
 * 8 g + 7]; i.e. W[n, k] sits at element
 *   ((n/16 * Kp/32 + k/32) * 64 + n%16 + 16 * ((k/8)%4)) * 8 + k%8.
 * W_rowmajor: device bf16 [N, ld], ld >= K; W_packed: device bf16, N * Kp
 * elements, not overlapping W_rowmajor.  N % 16 == 0, Kp % 128 == 0,
 * 0 < K <= Kp.  Errors: E_INVAL for shapes outside these rules or NULL. */
metro_status metro_op_pack_weight(const uint16_t* W_rowmajor, int32_t ld, int32_t N, int32_t K, int32_t Kp,
                                  uint16_t* W_packed, void* stream);

/* Projection GEMM of the Llama block (QKV, O, gate/up, down, LM head):
 *   acc[m, n] = sum_k X[m, k] * W[n, k]   (bf16 operands, fp32 accumulation)
 * X: bf16 [M, ldx] row-major, the first Kp columns used; W: bf16 [N, Kp] in
 * the layout metro_op_pack_weight writes; Kp % 128 == 0, N % 32 == 0,
 * ldx % 8 == 0; X, W, workspace and out_f32 16-byte aligned, out_bf16 8-byte
 * aligned (E_INVAL otherwise: the kernels move 16-byte pieces).
 * epilogue:
 *   0  out_f32[m*ldo + n]  = acc[m, n]
 *   1  out_f32[m*ldo + n] += acc[m, n]                       (residual add)
 *   2  W rows come in blocks of 16 = 8 gate rows then the 8 up rows of the
 *      same features (block b: gate_j, j = 8b .. 8b+7, then up_j);
 *      out_bf16[m*ldo + j] = bf16(silu(gate_j) * up_j), j < N/2
 *      (SwiGLU, Shazeer 2020).
 * workspace: NULL, or device fp32 [8][M][N]; when given, a decode-sized GEMM
 * (M <= 1024, epilogue 0 or 1) may run the k-split form the model uses (slices in
 * the workspace, then summed in slice order into the output), and a larger one
 * (any epilogue) may split the 256 x 256 tiles of its last, partly filled
 * round of workgroups over k the same way.  Its contents on return are
 * unspecified.
 * Errors: E_INVAL for shapes outside these rules or a NULL operand. */
metro_status metro_op_gemm(const uint16_t* X, int32_t ldx, const uint16_t* W, int32_t Kp, int32_t M, int32_t N,
                           int32_t epilogue, float* out_f32, uint16_t* out_bf16, int32_t ldo, float* workspace,
                           void* stream);

/* The kernels metro_op_gemm would run for a product (the model chooses by the
 * same rules), for inspection and tests; host only, no device work.
 * has_workspace: nonzero as for a non-NULL workspace.  *kind: 0 decode
 * kernel (weight streaming, up to 64 rows), 1 tiled with 128 x 128 blocks, 2
 * tiled with 256 (W rows) x 128 blocks, 3 tiled with 256 x 256 blocks, 4 tiled
 * with 128 x 64 blocks (33 to 64 rows).  Row strides of X that put the rows of a
 * block more than 4 GiB apart take the decode kernel whatever the kind, 64 rows
 * at a time and without k slices.  *k_slices:
 * k slices of every block (> 1 only with a workspace); *tail_split: k slices
 * of each block of the last, partly filled round of workgroups (1: none).
 * Counts compute units of the current device (256 when there is none).
 * Errors: E_INVAL (shape rules of metro_op_gemm, NULL outputs). */
metro_status metro_op_gemm_plan(int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t has_workspace,
                                int32_t* kind, int32_t* k_slices, int32_t* tail_split);

/* RMSNorm (Zhang & Sennrich 2019): h[r, :] = bf16(x[r, :] / sqrt(mean(x[r, :]^2)
 * + eps) * g), x fp32 [rows, d], g bf16 [d], h bf16 [rows, d], d % 4 == 0, d <= 8192;
 * x 16-byte aligned, g and h 8-byte aligned (E_INVAL otherwise). */
metro_status metro_op_rmsnorm(float* x, const uint16_t* g, float eps, uint16_t* h, int32_t rows, int32_t d,
                              void* stream);

/* Greedy choice: out[r] = lowest index of the maximum of logits[r, :] (fp32
 * [rows, vocab], vocab % 4 == 0); NaN values are skipped, -1 if none is left. */
metro_status metro_op_argmax(const float* logits, int32_t rows, int32_t vocab, int32_t* out, void* stream);

/* KV pages as the attention kernels read them (the layout of one layer's slab
 * of the model's pool): page p holds 16 consecutive positions; its bytes are
 * [K | V][kv_head][tile], a tile being 16 keys x head_dim bf16 in matrix-core
 * operand order:
 *   K tile:   key r, dim e  at ((e/32 * 4 + (e/8)%4) * 16 + r) * 8 + e%8
 *   V^T tile: dim e, key r  at ((e/32 * 4 + r/4) * 16 + e%16) * 8 + ((e/16)%2) * 4 + r%4
 * so that element (page, K|V = c, head h, ...) sits at
 *   page * (2 * n_kv_heads * 16 * head_dim) + (c * n_kv_heads + h) * 16 * head_dim + offset.
 * Page ids index this array (0 <= id < n_pages). */

/* Decode attention of the model's forward pass (grouped-query, causal, paged;
 * the attention of the Llama decoder the paper serves, §4.1): for each row i
 * and query head j, with kv head h = j / (nq / nkv) and keys t = 0 .. ctx[i]-1
 * of the row's pages,
 *   out[i, j, :] = bf16( sum_t softmax_t(q[i, j, :] . K[t, h, :] / sqrt(hd)) V[t, h, :] )
 * with fp32 scores, softmax and accumulation (the weights enter the bf16
 * matrix cores as a bf16 pair hi + lo).  Rows of more than 128 pages are cut
 * into 128-page work items whose states are merged in order, as in the model.
 *   q            device bf16 [rows, nq, hd], 16-byte aligned
 *   kv           device bf16, n_pages pages in the layout above, 16-byte aligned
 *   ctx          host int32 [rows], >= 1
 *   block_tables host int32, row after row: ceil(ctx[i] / 16) page ids each
 *   out          device bf16 [rows, nq * hd], 8-byte aligned
 * hd is 64 or 128; nq / nkv is 1, 2, 4 or 8.  Allocates and frees device
 * memory for its descriptors and split states and returns after the kernels
 * have finished on `stream` (a test entry point, not for serving loops).
 * Errors: E_INVAL (shapes, NULL, page id out of range), E_HIP. */
metro_status metro_op_attn_decode(const uint16_t* q, const uint16_t* kv, int32_t n_pages, int32_t nq, int32_t nkv,
                                  int32_t hd, int32_t rows, const int32_t* ctx, const int32_t* block_tables,
                                  uint16_t* out, void* stream);

/* Chunked-prefill attention of the model's forward pass: item i has
 * c_i = cu_q[i+1] - cu_q[i] queries (rows cu_q[i] .. cu_q[i+1]-1 of q and
 * out) at positions ctx_before[i] .. ctx_before[i] + c_i - 1, and its pages
 * hold keys 0 .. ctx_before[i] + c_i - 1 (the chunk's own keys included).
 * The query at position p sees keys 0 .. p (causal), otherwise as
 * metro_op_attn_decode.
 *   q            device bf16 [cu_q[n_items], nq, hd]
 *   cu_q         host int32 [n_items + 1], cu_q[0] = 0, each item >= 1 query
 *   ctx_before   host int32 [n_items], >= 0
 *   block_tables host int32, item after item: ceil((ctx_before[i] + c_i) / 16) ids
 *   out          device bf16 [cu_q[n_items], nq * hd]
 * Synchronous as metro_op_attn_decode.  Errors: E_INVAL, E_HIP. */
metro_status metro_op_attn_prefill(const uint16_t* q, const uint16_t* kv, int32_t n_pages, int32_t nq, int32_t nkv,
                                   int32_t hd, int32_t n_items, const int32_t* cu_q, const int32_t* ctx_before,
                                   const int32_t* block_tables, uint16_t* out, void* stream);

/* metro_op_attn_decode for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same kernels and results, with the descriptors and split
 * states in a fixed device array of 64 MiB that the library holds on each GPU
 * it runs on until the process ends, instead of a per-call allocation.  No
 * hipMalloc or hipFree, no allocating library call.  Arguments as for
 * metro_op_attn_decode (ctx and block_tables are host arrays, copied to the
 * device on `stream`).  Asynchronous: out is valid once `stream` has reached
 * the call.  Every call on one GPU uses that GPU's array, so calls that
 * overlap on one GPU (other streams or host threads) race; calls ordered on
 * one stream do not.  Needs 5 * rows + pages + 2 * work items int32 (each
 * rounded up to 256 bytes) plus work items * nkv * (nq / nkv) * (hd + 2) fp32,
 * a work item being up to 128 pages of one row.
 * Errors: E_INVAL as metro_op_attn_decode, E_CAPACITY when that exceeds the
 * array, E_HIP. */
metro_status metro_op_attn_decode_noalloc(const uint16_t* q, const uint16_t* kv, int32_t n_pages, int32_t nq,
                                          int32_t nkv, int32_t hd, int32_t rows, const int32_t* ctx,
                                          const int32_t* block_tables, uint16_t* out, void* stream);

/* --- 8-bit feed-forward: rows, weights and products of e4m3 values ----------
 *
 * 8-bit rows: row-major e4m3 codes (1 sign, 4 exponent, 3 mantissa bits; largest
 * finite value 448) [rows, ld], and for each 128 consecutive values of a row one
 * byte E in [rows, lds]: the values are code * 2^(E - 127).  A group's power of
 * two is the smallest that brings its largest magnitude within 448 (at least
 * 2^-126); codes are rounded from fp32 to nearest, ties to even.  An infinite or
 * NaN value becomes a NaN code; NaNs do not count for the power, an infinity
 * makes it 2^120.  Values behind the last column of a partly
 * filled group are zero codes; bytes of a row's stride behind its last group
 * are left as they were, and no result hangs on what they hold.
 *
 * The feed-forward block of a Llama layer in them: metro_op_rmsnorm_fp8,
 * metro_op_gemm_fp8 with gate and up (SwiGLU), metro_op_gemm_fp8 with down (bf16
 * rows, which the next layer's metro_op_rmsnorm_fp8 adds as its delta).  The
 * attention's output projection in bf16 weights adds itself to the residual
 * (metro_op_gemm, epilogue 1), and the norm behind it takes no delta.  By
 * experts: metro_op_rmsnorm_fp8 (with h_bf16), metro_op_gemm with the router's
 * weights, metro_op_route, metro_op_gemm_fp8_experts with gate and up and src,
 * the same with down, and metro_op_combine_experts.  Rows of a QKV product come
 * out plain; metro_op_rope_append turns them and writes the KV pages.
 *
 * All are asynchronous on `stream`, allocate nothing and may be captured into a
 * graph; a workspace belongs to one call at a time.  Calls of no rows (no tokens,
 * no slots) do nothing, metro_op_route aside, which writes empty experts; buffers
 * that would hold no element may be NULL. */

/* Weights of the 8-bit products.  The bf16 matrix W [N, Kp] (as for
 * metro_op_pack_weight: W[n, k] = W_rowmajor[n * ld + k] for k < K, 0 for K <= k <
 * Kp) in 8 bits, a power of two for each row's 128 columns, in matrix-core
 * operand order: code of W[n, k] at byte
 *   ((n/16 * Kp/128 + k/128) * 2 + (k/64)%2) * 1024 + (n%16 + 16 * ((k/16)%4)) * 16 + k%16
 * of W_packed (N * Kp bytes) and the byte E of row n, columns 128 b .. 128 b + 127 at
 *   ((n/16 * G/4 + b/4) * 16 + n%16) * 4 + b%4
 * of W_scale (N * G bytes), G = Kp / 128 rounded up to a multiple of 4.
 * W_packed and W_scale 16-byte aligned.  N % 16 == 0, Kp % 128 == 0, 0 < K <= Kp,
 * ld >= K.  Errors: E_INVAL. */
metro_status metro_op_pack_weight_fp8(const uint16_t* W_rowmajor, int32_t ld, int32_t N, int32_t K, int32_t Kp,
                                      uint8_t* W_packed, uint8_t* W_scale, void* stream);

/* Residual addition, RMSNorm and 8-bit rows in one pass over the residual:
 *   x'[r, :] = x[r, :] + delta[r, :]                  (x where delta is NULL)
 *   v[r, :]  = x'[r, :] / sqrt(mean(x'[r, :]^2) + eps) * g
 * in fp32, the sum of the squares too (a row whose sum passes it has v = 0).
 * h, h_scale <- v as 8-bit rows; h_bf16 <- bf16(v) unless NULL; x_out <- x'
 * unless NULL (x_out only with delta; it may be x).
 *   x, x_out  fp32 [rows, ldx], 16-byte aligned, ldx % 4 == 0
 *   delta     bf16 [rows, ldd] or NULL, 8-byte aligned, ldd % 4 == 0
 *   g         bf16 [d], 8-byte aligned
 *   h_bf16    bf16 [rows, ldh_bf16] or NULL, 8-byte aligned, ldh_bf16 % 4 == 0
 *   h         e4m3 [rows, ldh], 4-byte aligned, ldh % 4 == 0, at least d rounded up to 128
 *   h_scale   [rows, lds], lds >= ceil(d / 128)
 * (metro_op_gemm_fp8 reads h with 16-byte alignment, ldh % 16 == 0, and lds % 4
 * == 0.)  d % 4 == 0, d <= 8192.  Errors: E_INVAL. */
metro_status metro_op_rmsnorm_fp8(const float* x, int32_t ldx, const uint16_t* delta, int32_t ldd, const uint16_t* g,
                                  float eps, float* x_out, uint16_t* h_bf16, int32_t ldh_bf16, uint8_t* h, int32_t ldh,
                                  uint8_t* h_scale, int32_t lds, int32_t rows, int32_t d, void* stream);

/* Product of 8-bit rows and weights:
 *   acc[m, n] = sum_b 2^(Ex[m, b] + Ew[n, b] - 254) * sum_{k in b} X[m, k] * W[n, k]
 * with fp32 accumulators.  (The matrix cores align the products of each eight
 * columns to the largest and cut the others below 2^-13 of it: at most 7 * 2^-13 of
 * sum_k |x w|, 1.5e-5 of the result's 2-norm on normal data.)
 *   X, x_scale  8-bit rows [M, ldx], [M, ldxs]: the first Kp columns; X 16-byte
 *               aligned, ldx % 16 == 0; x_scale 4-byte aligned, ldxs % 4 == 0,
 *               ldxs >= Kp / 128 rounded up to 4
 *   W, w_scale  as metro_op_pack_weight_fp8 writes them, 16-byte aligned
 * Kp % 128 == 0, N % 32 == 0, M <= 2^26, N <= 2^30, M * N <= 2^36.  epilogue:
 *   0  out_bf16[m*ldo + n] = bf16(acc[m, n]); 8-byte aligned, ldo % 4 == 0, ldo >= N
 *   2  W rows in blocks of 16 = 8 gate rows then the 8 up rows of the same
 *      features (as metro_op_gemm): silu(gate) * up as 8-bit rows of N / 2 values
 *      in out_fp8 [M, ldo] (16-byte aligned, ldo % 16 == 0, ldo >= N / 2 rounded up
 *      to 128) and out_scale [M, ldos] (ldos >= ceil(N / 256)), rounded from fp32;
 *      silu(gate) is 0 for gates below -87.33, whose sigmoid is below 2^-126
 * The other output is NULL.
 * workspace: NULL, or device fp32 of workspace_bytes, 16-byte aligned: small
 * products may then run as k slices (ks * M * N floats for ks <= 8 slices where
 * they fit), summed in slice order.  Which slices run follows from the sizes and
 * workspace_bytes, so results of equal calls are equal bit for bit.  Outputs
 * overlap no input.  Errors: E_INVAL. */
metro_status metro_op_gemm_fp8(const uint8_t* X, int32_t ldx, const uint8_t* x_scale, int32_t ldxs, const uint8_t* W,
                               const uint8_t* w_scale, int32_t Kp, int32_t M, int32_t N, int32_t epilogue,
                               uint16_t* out_bf16, uint8_t* out_fp8, int32_t ldo, uint8_t* out_scale, int32_t ldos,
                               float* workspace, int64_t workspace_bytes, void* stream);

/* What metro_op_gemm_fp8 (n_experts 0) or metro_op_gemm_fp8_experts (M slots; X
 * gathered or not, its rows and their powers within 4 GiB) would run, for
 * inspection and tests; host only, no device work.  *kind: 0 direct (operands
 * beyond the others' 32-bit offsets), 1 streaming, 2 tiled.  *w_rows, *x_rows:
 * rows of W and of X of a workgroup.  *k_slices: slices that a finishing
 * launch sums, 0: none.  Errors: E_INVAL (shape rules of metro_op_gemm_fp8,
 * NULL outputs). */
metro_status metro_op_gemm_fp8_plan(int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t n_experts,
                                    int64_t workspace_bytes, int32_t* kind, int32_t* w_rows, int32_t* x_rows,
                                    int32_t* k_slices);

/* Whether that product's weights would pass the caches by (*w_bypass 1, else 0):
 * such kernels are built apart, so tests of every variant need to tell them.
 * Host only; arguments and errors as metro_op_gemm_fp8_plan. */
metro_status metro_op_gemm_fp8_plan_bypass(int32_t M, int32_t N, int32_t Kp, int32_t epilogue, int32_t n_experts,
                                           int64_t workspace_bytes, int32_t* w_bypass);

/* Routing of T tokens to top_k of n_experts experts each.  With z = logits[t, :]
 * and, in fp64, s = softmax(z) (scoring 0) or 1 / (1 + exp(-z)) (scoring 1):
 *   choice c = s + bias (bias fp32 [n_experts] or NULL; -inf shuts an expert out)
 *   experts in n_groups equal runs; a group's score is the sum of its two largest
 *   c among the open experts (its one c where one is open, behind every other
 *   group where none is); the top_groups best groups stay
 *   experts[t, :]  the top_k largest c of theirs, largest first
 *   weights[t, :]  their s * scale, with renormalise s / sum of the top_k s * scale
 *                  (0 where that sum is 0)
 * Ties go to the lowest index.  A NaN choice counts as -inf: where too few open
 * experts are left, the lowest indices of the staying groups are chosen, so
 * indices are always distinct and in range.  An expert that its bias shuts out
 * has s = 0 among the weights then.  A row of -inf has s = 0; a NaN or +inf in a
 * softmax row makes its weights NaN (those of shut out experts may stay 0).
 * And the experts' order of the T * top_k rows, tokens ascending within an expert:
 *   offsets [n_experts + 1]: expert e has slots offsets[e] .. offsets[e + 1] - 1
 *   src  [T * top_k]: token of a slot;  slot [T, top_k]: slot of a choice
 *   logits    device fp32 [T, ldl], ldl >= n_experts (metro_op_gemm's output with
 *             the router's rows padded to 32 will do)
 *   experts, src, slot, offsets  device int32;  weights  device fp32
 *   workspace device int32 of at least 4 * n_experts * ceil(T / 64) bytes; may be
 *             NULL for T <= 64
 * 1 <= n_experts <= 512, 1 <= n_groups <= 64, top_k <= 32 and at most the experts of
 * top_groups groups, T <= 2^24.  Errors: E_INVAL. */
metro_status metro_op_route(const float* logits, int32_t ldl, const float* bias, int32_t T, int32_t n_experts,
                            int32_t scoring, int32_t n_groups, int32_t top_groups, int32_t top_k, int32_t renormalise,
                            float scale, int32_t* experts, float* weights, int32_t* offsets, int32_t* src, int32_t* slot,
                            int32_t* workspace, int64_t workspace_bytes, void* stream);

/* metro_op_gemm_fp8 by experts: slot m (0 <= m < R) of expert e, offsets[e] <= m <
 * offsets[e + 1], is row src[m] of X (row m with src NULL) times expert e's weights,
 *   W + e * N * Kp, w_scale + e * N * G  (each as metro_op_pack_weight_fp8 writes it).
 *   src       device int32 [R] or NULL: 0 <= src[m] < x_rows
 *   offsets   device int32 [n_experts + 1], ascending, 0 <= offsets[e] <= R (as
 *             metro_op_route leaves them)
 *   x_rows    rows of X; at least R with src NULL
 * Both are read on the device and held to these ranges there: a row index
 * outside reads another row of X, and nothing outside the buffers is touched.
 * Output rows of slots that no expert has are left as they were.  Shapes,
 * epilogues, alignments, workspace and precision as metro_op_gemm_fp8, with R in
 * the place of M; n_experts <= 1024.  Errors: E_INVAL. */
metro_status metro_op_gemm_fp8_experts(const uint8_t* X, int32_t ldx, const uint8_t* x_scale, int32_t ldxs,
                                       int32_t x_rows, const int32_t* src, const int32_t* offsets, int32_t n_experts,
                                       int32_t R, const uint8_t* W, const uint8_t* w_scale, int32_t Kp, int32_t N,
                                       int32_t epilogue, uint16_t* out_bf16, uint8_t* out_fp8, int32_t ldo,
                                       uint8_t* out_scale, int32_t ldos, float* workspace, int64_t workspace_bytes,
                                       void* stream);

/* The experts' rows back at their tokens:
 *   out[t, :] = resid[t, :] + sum_j weights[t, j] * y[slot[t, j], :]   (fp32, j ascending)
 * A slot outside 0 .. y_rows - 1 adds nothing (a choice that was dropped).
 *   y         device bf16 [y_rows, ldy], 16-byte aligned, ldy % 8 == 0
 *   weights, slot  device fp32, int32 [T, top_k]
 *   resid     device fp32 [T, ldo] or NULL (0), 16-byte aligned; may be out
 *   out       device fp32 [T, ldo], 16-byte aligned, ldo % 4 == 0
 * d % 8 == 0.  Errors: E_INVAL. */
metro_status metro_op_combine_experts(const uint16_t* y, int32_t ldy, int32_t y_rows, const float* weights,
                                      const int32_t* slot, int32_t T, int32_t top_k, int32_t d, const float* resid,
                                      float* out, int32_t ldo, void* stream);

/* --- a speculative decoding step ---------------------------------------------
 *
 * What a layer does with rows of a QKV product, for callers that run layers of
 * their own (metro_op_gemm, metro_op_gemm_fp8) over pages of the layout above:
 * metro_op_rope_append puts the drafted tokens' keys and values into the cache and
 * leaves their queries, metro_op_attn_tree attends over both, and behind the
 * head's product metro_op_sample chooses a token at every drafted one.  The
 * drafts whose tokens agree are accepted; metro_op_kv_move brings their keys and
 * values, in all layers, to the slots behind the context.  One token a sequence
 * without drafts is the case of one query an item, a prompt's chunk that of a
 * chain of them (whose keys behind a query are read as well: a chunk of hundreds of
 * tokens without context takes 2 to 5 times as long as metro_op_attn_prefill's
 * kernel, one of 512 behind 4096 keys about the same).
 *
 * All are asynchronous on `stream`, allocate nothing and may be captured into a
 * graph; a workspace belongs to one call at a time.  Calls of no rows (items,
 * moves) do nothing; buffers that would hold no element may be NULL.  Index arrays
 * are read on the device and held to their ranges there: an index outside touches
 * nothing outside the buffers. */

/* Rows of a QKV product into the cache.  Of row t, head by head (nq query heads,
 * nkv key heads, nkv value heads of hd columns each, in plain order):
 *   y <- y / sqrt(mean(y^2) + eps) * gain     query heads with q_gain, key heads
 *                                             with k_gain (NULL: no norm)
 *   (y_i, y_{i+hd/2}) <- (y_i c - y_{i+hd/2} s, y_i s + y_{i+hd/2} c),  i < hd/2,
 *                  (c, s) = rope[pos[t], i]   query and key heads
 * in fp32, the sum of the squares too (a head whose sum passes it comes out as 0),
 * rounded to bf16 once: queries to q[t], keys and values to the cache's slot[t]
 * (page * 16 + offset).  A row whose slot lies outside 0 .. 16 n_pages - 1
 * (a padded batch's) leaves the cache as it is, its queries are written all the
 * same.  A position outside 0 .. n_pos - 1 makes the row's queries and keys NaN.
 * Slots of different rows differ; of rows with the same slot the cache keeps
 * values of one or the other.
 *   qkv_f32, qkv_bf16  device [T, ld], one of them, the other NULL; 16-byte aligned,
 *             ld % 8 == 0, ld >= (nq + 2 nkv) hd
 *   q_gain, k_gain  device bf16 [hd] or NULL, 16-byte aligned
 *   rope      device fp32 [n_pos, hd / 2, 2], 16-byte aligned
 *   pos, slot device int32 [T]
 *   q         device bf16 [T, nq, hd], 16-byte aligned
 *   kv        device bf16, n_pages pages in the layout above, 16-byte aligned
 * Outputs overlap no input.  hd 64 or 128, nq <= 1024, nkv <= 256, T * (nq + 2 nkv)
 * <= 2^25, n_pages < 2^27.  Errors: E_INVAL. */
metro_status metro_op_rope_append(const float* qkv_f32, const uint16_t* qkv_bf16, int32_t ld, int32_t T, int32_t nq,
                                  int32_t nkv, int32_t hd, const uint16_t* q_gain, const uint16_t* k_gain, float eps,
                                  const float* rope, int32_t n_pos, const int32_t* pos, const int32_t* slot, uint16_t* q,
                                  uint16_t* kv, int32_t n_pages, void* stream);

/* Keys and values from slot to slot of the cache, in n_layers layers whose pages
 * lie layer_stride elements apart: for each group g of moves and j = offsets[g] ..
 * offsets[g+1] - 1 in order, dst[j] <- src[j], as if all sources of a group were
 * read before its first destination is written.  Groups of more than 8 moves go 8
 * at a time, in order, which is the same where no move of an earlier 8 writes a
 * later one's source: so for an accepted path, listed in the order of its tokens and
 * brought to places at or before theirs in the sequence, in whatever order the
 * sequence's pages have their ids.  A later move of a group to the same slot wins.
 * A slot that one group writes is neither read nor written by another.  Moves from
 * or to a slot outside 0 .. 16 n_pages - 1 are left out.
 *   kv        device bf16, 16-byte aligned; layer_stride % 8 == 0, at least n_pages
 *             pages (not looked at for one layer)
 *   src, dst  device int32 [n_moves];  offsets  device int32 [n_groups + 1],
 *             ascending, within 0 .. n_moves
 * hd 64 or 128, nkv <= 256, n_layers and n_groups <= 65535.  Errors: E_INVAL. */
metro_status metro_op_kv_move(uint16_t* kv, int64_t layer_stride, int32_t n_layers, int32_t n_pages, int32_t nkv, int32_t hd,
                              const int32_t* src, const int32_t* dst, const int32_t* offsets, int32_t n_groups,
                              int32_t n_moves, void* stream);

/* Attention of drafted tokens over the cache.  Item i has the query rows cu_q[i] ..
 * cu_q[i+1] - 1, n of them, and its pages hold keys 0 .. ctx[i] + n - 1, the last n
 * those of the queries in their order.  Query r of the item sees keys 0 .. ctx[i] -
 * 1 and key ctx[i] + j where bit j % 32 of mask[row, j / 32] is set (mask NULL: for
 * j <= r, a chain); over the keys t that it sees, as metro_op_attn_decode,
 *   out[row, head, :] = bf16( sum_t softmax_t(q . K[t] / sqrt(hd)) V[t] ),
 * zeros where it sees none, or none whose score is above -inf.  Sums are fp32 and
 * divided at the end: values up to 2^89 in magnitude stay finite.  What the keys that
 * a query does not see hold (NaN, Inf) does not reach it; an infinity among the
 * values of the ctx keys makes its outputs infinite or NaN.  Rows in no item are
 * left as they were.
 *   q         device bf16 [rows, nq, hd], 16-byte aligned
 *   kv        device bf16, n_pages pages in the layout above, 16-byte aligned
 *   cu_q      device int32 [n_items + 1], ascending, within 0 .. rows
 *   ctx       device int32 [n_items], >= 0
 *   max_q     most queries of an item, 1 .. 4096; later ones are left as they were
 *   max_keys  most keys of an item (ctx + its queries), 1 .. 2^30; keys from there
 *             on are not seen.  The larger it is beside the items' own, the fewer workgroups
 *             share the keys there are
 *   mask      device uint32 [rows, ldm] or NULL, 32 * ldm >= max_q
 *   block_tables  device int32 [n_items, ldb] page ids, 16 * ldb >= max_keys
 *   out       device bf16 [rows, nq * hd], 16-byte aligned, not q
 *   workspace NULL, or device fp32 of workspace_bytes, 16-byte aligned: what
 *             metro_op_attn_tree_workspace says lets the keys of an item be split
 *             over workgroups as the call's size asks for, less gives fewer splits,
 *             NULL none.  Which splits run follows from the sizes and
 *             workspace_bytes, and their states are merged in order, so results of
 *             equal calls are equal bit for bit
 * hd 64 or 128, nq / nkv 1, 2, 4 or 8, nkv <= 256, n_items * max_q <= 2^22 and
 * n_items * nkv * ceil(max_q * nq / nkv / 16) <= 2^22.  Errors: E_INVAL. */
metro_status metro_op_attn_tree(const uint16_t* q, const uint16_t* kv, int32_t n_pages, int32_t nq, int32_t nkv, int32_t hd,
                                int32_t n_items, const int32_t* cu_q, int32_t rows, const int32_t* ctx, int32_t max_q,
                                int32_t max_keys, const uint32_t* mask, int32_t ldm, const int32_t* block_tables,
                                int32_t ldb, uint16_t* out, float* workspace, int64_t workspace_bytes, void* stream);

/* *bytes: the workspace that metro_op_attn_tree makes use of; host only. */
metro_status metro_op_attn_tree_workspace(int32_t nq, int32_t nkv, int32_t hd, int32_t n_items, int32_t rows, int32_t max_q,
                                          int32_t max_keys, int64_t* bytes);

/* Sampled choice of a token of each row.  With x = logits[r, 0 .. vocab - 1], the
 * tokens in the order of falling x, ties by rising index, and in fp64
 *   w = exp((x - max x) / temperature[r])        (1 where x is the largest)
 *   min-p  keeps the tokens with w >= min_p[r]   (<= 0: all; >= 1: those of w = 1)
 *   top-k  keeps the first top_k[r] of them      (<= 0: all)
 *   top-p  keeps the shortest beginning of them whose sum of w is at least top_p[r]
 *          of theirs, one token at the least     (>= 1: all)
 *   out[r] = the first token of the order whose sum of w up to and with it is above
 *          u[r] times the sum of the kept ones
 *   prob[r] = its w / that sum, unless prob is NULL
 * so u = 0 gives the most likely token, and u uniform on [0, 1) samples.  u below 0
 * or NaN counts as 0, from 1 on it gives the last kept token, however little its
 * weight adds to the sum.  Weights are held to 2^-35 of themselves (to 2^-51 |x /
 * temperature|, where that is more); tokens whose weights lie below 2^-46 may count
 * as not there (of 2^18 they change the sums by less than 2^-28).  temperature 0,
 * below 0 or NaN is the greedy choice (metro_op_argmax, prob 1).  A NaN setting
 * otherwise counts as not set; a NULL array sets none (temperature 1).  NaN logits
 * are skipped; out is -1 and prob 0 where none is above -inf.
 *   logits  device fp32 [rows, ldl], ldl >= vocab
 *   temperature, top_p, min_p, u  device fp32 [rows];  top_k, out  device int32 [rows]
 *   prob    device fp32 [rows] or NULL
 *   workspace  device, 16-byte aligned, of at least what metro_op_sample_workspace says
 * Results do not depend on the order in which anything is added.  vocab <= 2^18, rows
 * <= 65535.  Errors: E_INVAL. */
metro_status metro_op_sample(const float* logits, int32_t ldl, int32_t rows, int32_t vocab, const float* temperature,
                             const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* out,
                             float* prob, void* workspace, int64_t workspace_bytes, void* stream);

/* *bytes: the workspace that metro_op_sample needs; host only. */
metro_status metro_op_sample_workspace(int32_t rows, int32_t vocab, int64_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* METRO_OPS_H */
