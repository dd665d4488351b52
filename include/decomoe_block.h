/*
 * decomoe_block.h - C ABI of the attention half of a decoder block on the
 * MI355X (gfx950): what stands between two MoE layers (decomoe.h) when a
 * model decodes over a paged key/value cache.
 *
 *   RMS norm with the residual's addition, 16-bit or 8-bit output  blk_rms_norm
 *   page tables and slot maps from request lengths                  blk_kv_extend
 *   head norm, rotation, and the write into the paged cache         blk_qkv_cache
 *   attention of one new token a sequence over its pages            blk_attn_decode
 *   products of few rows with 4-bit weights                         blk_linear_w4
 *   4-bit weights from float ones (once, at load time)              blk_quantize_w4
 *
 * A decode step calls blk_kv_extend once and then, per layer,
 *   blk_rms_norm (8-bit out) -> blk_linear_w4 (q, k, v) -> blk_qkv_cache
 *   -> blk_attn_decode -> blk_linear_w4 (output projection)
 *   -> blk_rms_norm (residual) -> moe_rcep_layer(x = y, residual = h, out = h).
 *
 * The library is libdecomoe_block.so.  Status codes and moe_dtype are those
 * of decomoe.h (moe_status_string gives their texts), and so are its
 * conventions: device pointers owned by the caller, contiguous row-major
 * arrays at 16-byte aligned addresses, host-side checks before anything is
 * launched, asynchronous calls on `stream` on the current HIP device, no
 * allocation and no synchronisation, outputs that do not overlap inputs or
 * each other except where stated, and bitwise the same results from run to
 * run.  Contents of device arrays are not checked on the host; the kernels
 * skip entries that are out of range as stated, so that no access leaves its
 * array.  Every call can be captured into a HIP graph.
 *
 * 8-bit rows (BLK_MX8): OCP microscaling.  A row of n values is n e4m3 bytes
 * and ceil(n / 32) scale bytes (e8m0: byte b stands for 2^(b - 127), 255 for
 * NaN), one for every 32 consecutive values.  Where this library makes them,
 * the scale is the smallest 2^E, E >= -127, with max |v| <= 448 * 2^E, and
 * each value is v * 2^-E rounded to the nearest e4m3 value, ties to even (so
 * nothing saturates).  A block that holds an infinity or a NaN gets the
 * scale byte 255 and stands for NaNs.
 * 4-bit weights: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives
 * from code 8 on), two to a byte, the even column in the low half, with the
 * same scale bytes for every 32 columns of a row.
 */
#ifndef DECOMOE_BLOCK_H
#define DECOMOE_BLOCK_H

#include "decomoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dtype of 8-bit rows, where a function takes it beside MOE_F32 and MOE_BF16 */
#define BLK_MX8 2

/*
 * blk_rms_norm - h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight.
 *
 *   x, residual  [T, d] (dtype); residual may be NULL (then h = x).
 *   weight       [d] float32, or NULL (ones).
 *   h_out        [T, d] (dtype) or NULL: h, rounded once.
 *   y            [T, d] (dtype) or NULL: y, rounded once.
 *   q, q_scale   [T, d] e4m3 and [T, ceil(d / 32)] scale bytes, or both
 *                NULL: y as 8-bit rows, from the unrounded y.
 * At least one of h_out, y and q must be given.  h and y are formed in
 * float32, the row's sum and mean in 64 bits, from the unrounded h (squares
 * that float32 does not hold are taken in 64 bits, so y is right for every
 * finite h).  h_out
 * or y may be x or residual themselves (not both the same array); any other
 * overlap is MOE_EALIAS.
 * Limits: 1 <= d <= 32768, eps >= 0; T >= 0, at most 2^25 (d > 512: 2^23,
 * d > 4096: 2^21).
 */
int blk_rms_norm(const void* x, moe_dtype dtype, const void* residual, const float* weight, int T, int d, double eps,
                 void* h_out, void* y, void* q, uint8_t* q_scale, hipStream_t stream);

/*
 * blk_kv_extend - the page tables and the slot map of a step's new tokens,
 * and the pages of finished sequences, from the request lengths alone.
 *
 * A cache of n_pages pages of page_size slots is shared by n_seq sequences.
 * Slot page * page_size + i is token i of a page.  Sequence s holds
 * ceil(len[s] / page_size) pages, the first entries of its table row.
 *
 *   len_in       [n_seq] tokens of each sequence in the cache.
 *   add          [n_seq] tokens to append (>= 0), or negative: the sequence
 *                is finished and gives its pages back.
 *   n_free_in    [1] pages on the stack of free ones.
 *   free_pages   [n_pages] in and out: the stack; entries [0, n_free) are free.
 *   block_table  [n_seq, max_pages] in and out: page indices; only the
 *                entries of newly taken pages are written.
 *   len_out      [n_seq] lengths afterwards (0 for a finished sequence).
 *   n_free_out   [1].
 *   row_offsets  [n_seq + 1] exclusive sums of the appended tokens: rows
 *                [row_offsets[s], row_offsets[s + 1]) of the step's batch are
 *                sequence s's, in order (clamped to rows_max).
 *   slot_map     [rows_max] slot of each row; -1 where nothing may be written:
 *                rows behind the last sequence and rows of refused ones.
 *   positions    [rows_max] index of each row in its sequence (0 with slot -1).
 *   accepted     [n_seq] 1 where the request was carried out, 0 where refused.
 *   status       [4] rows, pages taken, sequences refused, pages given back.
 * Finished sequences come first: their pages go onto the stack in sequence
 * order and table order.  Then pages are taken from the top of the stack in
 * sequence order.  A sequence is refused - it keeps its length and takes
 * nothing - when its tokens do not fit max_pages pages or its rows end behind
 * rows_max, or when it needs pages and the pages needed up to it (by it and
 * by the sequences before it that pass those two tests) are more than there
 * are.  len_out may be len_in and n_free_out may be n_free_in (a captured
 * step that advances itself).
 * Lengths outside [0, max_pages * page_size] and free counts outside
 * [0, n_pages] are clamped; a page index outside [0, n_pages) yields slot -1.
 * Limits: n_seq >= 0, page_size >= 1, n_pages >= 1, max_pages >= 1,
 * rows_max >= 0; n_pages * page_size and max_pages * page_size at most
 * INT32_MAX, n_seq * max_pages and rows_max at most 2^30 (else
 * MOE_EUNSUPPORTED).
 */
int blk_kv_extend(const int32_t* len_in, const int32_t* add, int n_seq, int page_size, int max_pages, int n_pages,
                  int rows_max, const int32_t* n_free_in, int32_t* block_table, int32_t* free_pages,
                  int32_t* len_out, int32_t* n_free_out, int32_t* row_offsets, int32_t* slot_map,
                  int32_t* positions, int32_t* accepted, int32_t* status, hipStream_t stream);

/*
 * blk_qkv_cache - the heads of T rows: RMS norm and rotation of the query
 * and key heads, and the write of keys and values into the paged cache.
 *
 *   qkv         [T, n_q + 2 n_kv, D] (dtype): query, key and value heads.
 *   q_norm,
 *   k_norm      [D] float32 or NULL: weights of the norm over each query /
 *               key head, v / sqrt(mean(v^2) + eps) * weight (NULL: no norm).
 *   positions   [T] int32; inv_freq [rot / 2] float32: with rot > 0, values
 *               i and i + rot / 2 of a query or key head, i < rot / 2, are
 *               rotated by the angle positions[t] * inv_freq[i] (formed in
 *               64 bits); values from rot on are left as they are.  rot = 0:
 *               no rotation, both may be NULL.
 *   slot_map    [T] int32 slots; rows with a slot outside
 *               [0, n_pages * page_size) are not written to the cache.  The
 *               other slots must be distinct: of a slot given twice each
 *               value is one of the two rows'.
 *   q_out       [T, n_q, D] (dtype).
 *   k_cache,
 *   v_cache     [n_pages, n_kv, page_size, D] of cache_dtype: dtype itself,
 *               or BLK_MX8 (bf16 rows) with
 *   k_scale,
 *   v_scale     [n_pages, n_kv, page_size, D / 32] (else NULL).
 * Every other slot of the cache is left as it was.  Values are formed in
 * float32 (with the values of a head whose squares it does not hold brought to
 * the middle of its range) and rounded once.
 * Limits: D % 32 == 0, 32 <= D <= 256; rot % 16 == 0, 0 <= rot <= D; n_q,
 * n_kv from 1 to 16384; 0 <= T <= 2^25; page_size, n_pages >= 1; n_pages * page_size <= INT32_MAX;
 * eps >= 0 (sizes this library does not take: MOE_EUNSUPPORTED).
 */
int blk_qkv_cache(const void* qkv, moe_dtype dtype, int T, int n_q, int n_kv, int D, const float* q_norm,
                  const float* k_norm, double eps, const int32_t* positions, const float* inv_freq, int rot,
                  const int32_t* slot_map, int cache_dtype, int n_pages, int page_size, void* q_out, void* k_cache,
                  void* v_cache, uint8_t* k_scale, uint8_t* v_scale, hipStream_t stream);

/*
 * blk_attn_decode - attention of one new token of each sequence over its
 * pages: out[s, h] = sum_j softmax_j(scale * q[s, h] . k_j) v_j over the keys
 * j < lens[s] of key/value head h / (n_q / n_kv).
 *
 *   q            [n_seq, n_q, D] (dtype).
 *   k_cache .. v_scale  as in blk_qkv_cache (n_kv heads; cache_dtype dtype,
 *                or BLK_MX8 with bf16 q).
 *   block_table  [n_seq, max_pages] int32; lens [n_seq] int32 keys of each
 *                sequence, the new token's own included (clamped to
 *                [0, max_pages * page_size]).
 *   out          [n_seq, n_q, D] (dtype).
 * A sequence without keys, and one all of whose scores are minus infinity,
 * gives zeros.  Keys on a page outside [0, n_pages) are left out.  What the
 * cache holds in slots behind a sequence's last key is never used.
 * Products are accumulated in float32 with a running float32 maximum and sum
 * per head.  bf16: the softmax terms enter the product with v in two bf16
 * parts (2^-16 of a term is lost at most).  8-bit keys and values are used as
 * bf16, which holds them exactly from 2^-133 to below 2^128 (all of scale
 * bytes 3 to 246; larger ones are infinities).
 * Needs ws of blk_attn_workspace_size(n_seq, n_q, n_kv, D,
 * max_pages * page_size) bytes; its contents need no initialisation.
 * Limits: D in {32, 64, 96, 128, 192, 256}; n_q % n_kv == 0; n_seq <= 4096;
 * n_seq * n_kv * ceil(n_q / n_kv / 16) <= 2^23; scale * log2(e) finite in
 * float32; n_pages * n_kv * page_size < 2^32 - 1, max_pages * page_size <= 2^30 and
 * n_seq * max_pages * page_size * n_kv * ceil(n_q / n_kv / 16) / 64 below
 * 2^31 (else MOE_EUNSUPPORTED; blk_attn_workspace_size returns 0 for sizes
 * that are not taken).
 */
size_t blk_attn_workspace_size(int n_seq, int n_q, int n_kv, int D, int max_keys);
int blk_attn_decode(const void* q, moe_dtype dtype, int n_seq, int n_q, int n_kv, int D, const void* k_cache,
                    const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int cache_dtype,
                    int n_pages, int page_size, const int32_t* block_table, int max_pages, const int32_t* lens,
                    double scale, void* out, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * blk_linear_w4 - y[t, r] = sum_c x[t, c] * w[r, c] with 4-bit weights.
 *
 *   x        [T, k] of x_dtype: MOE_BF16, MOE_F32, or BLK_MX8 with
 *   x_scale  [T, k / 32] scale bytes (else NULL).
 *   codes    [n, k / 2] and scales [n, k / 32]: the weights (row-major, as
 *            4-bit weights are stored and exchanged; no re-layout).
 *   y        [T, n] of y_dtype (MOE_BF16 or MOE_F32), rounded once.
 * bf16 x: exact products on the bf16 matrix instructions, accumulated in
 * float32; float32 x: float32 matrix instructions (in both, weights of 2^128
 * and more, which scale bytes 253 and 254 can give, are infinities).  8-bit x:
 * the scaled 8-bit by 4-bit matrix instruction, which aligns the exact products of eight
 * neighbouring columns to the largest of them and keeps 13 bits below its
 * exponent (each of the others loses less than 2^-13 of the largest, next to
 * the 2^-4 that a value lost when it became e4m3), then adds in float32.
 * Made for few rows (decode steps): beyond 64 rows the weights are read again
 * for every 64.
 * Limits: 0 <= T <= 2^22, 1 <= n <= 2^26, 32 <= k <= 2^24, k % 32 == 0.
 */
int blk_linear_w4(const void* x, int x_dtype, const uint8_t* x_scale, int T, int k, const uint8_t* codes,
                  const uint8_t* scales, int n, void* y, moe_dtype y_dtype, hipStream_t stream);

/*
 * blk_quantize_w4 - 4-bit weights of float ones, once when a layer is loaded.
 *
 *   w       [n, k] (dtype).
 *   codes   [n, k / 2], scales [n, k / 32]: for every 32 columns the smallest
 *           2^E, E >= -127, with max |w| <= 6 * 2^E, and w * 2^-E rounded to
 *           the nearest e2m1 value, ties to the even code.  A block that holds
 *           an infinity or a NaN gets the scale byte 255.
 * Limits: n >= 1, k >= 32, k % 32 == 0.
 */
int blk_quantize_w4(const void* w, moe_dtype dtype, int n, int k, uint8_t* codes, uint8_t* scales,
                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DECOMOE_BLOCK_H */
