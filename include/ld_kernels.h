/*
 * libld, kernel-level entry points: each step of the decode / prefill pass as a call of its
 * own, so that tests and micro-benchmarks can drive one kernel at a time.  ld_prefill /
 * ld_decode_step / ld_step_mixed are compositions of exactly these launches.
 *
 * All data pointers are DEVICE pointers owned by the caller unless marked HOST.  `stream`
 * is a hipStream_t as void*.  Calls only enqueue work; they return LD_E_INVAL for
 * unsupported shapes (before launching anything) and LD_E_HIP if the launch failed.
 * Activations are float32 throughout; `dtype` (LD_F32 | LD_BF16) is the element type of
 * matrices and of the KV pool.
 */
#ifndef LD_KERNELS_H
#define LD_KERNELS_H

#include "ld.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { LDK_STORE = 0, LDK_ADD = 1, LDK_SWIGLU = 2 };

/* x[t, :] = embed[tok[t], :] widened to float32.  tok values must be < vocab (checked by the
 * caller of the step functions on the host). */
ld_status ldk_embed(const void *embed, int32_t dtype, const int32_t *tok, int32_t T, int32_t d, float *x,
                    void *stream);

/* out[r, i] = x[row, i] / sqrt(mean_j x[row, j]^2 + eps) * g[i], row = row_idx ? row_idx[r] : r. */
ld_status ldk_rmsnorm(const float *x, const float *g, const int32_t *row_idx, int32_t R, int32_t d, float eps,
                      float *out, void *stream);

/* Scratch bytes ldk_linear (ldk_qkv_rope: epilogue LDK_STORE, N = (H + 2 Hkv) hd) can use for T rows
 * (0 for T < 2): the two-part bf16 image of the input plus split-K partial sums. */
size_t ldk_linear_scratch_bytes(int32_t T, int32_t N, int32_t K, int32_t epilogue);

/* Linear layer on T rows: acc[t, n] = sum_k W[n, k] x[t, k], float32 accumulation.
 *   LDK_STORE : y[t, n]  = acc[t, n]                          W [N, K]
 *   LDK_ADD   : y[t, n] += acc[t, n]   (residual)             W [N, K]
 *   LDK_SWIGLU: y[t, n]  = silu(acc[t, n]) * acc[t, N + n]    W [2N, K]  (gate rows, then up rows)
 * If g != NULL the input is RMS-normalised on the fly: x[t, k] is replaced by
 * x[t, k] * rsqrt(mean_k x[t, k]^2 + eps) * g[k].
 * x [T, K], y [T, N] dense row-major.  K must be a multiple of 8.
 * Kernel choice: one bf16 row -> bandwidth-bound matrix-vector kernel; several bf16 rows with
 * K a multiple of 128 and scratch of ldk_linear_scratch_bytes(...) bytes -> matrix cores
 * (activations split into two bf16 parts, float32 accumulation); otherwise (float32 matrices, no
 * scratch) a plain vector-ALU kernel.  scratch may be NULL. */
ld_status ldk_linear(const void *W, int32_t dtype, const float *x, const float *g, float eps, int32_t T,
                     int32_t N, int32_t K, int32_t epilogue, float *y, void *scratch, size_t scratch_bytes,
                     void *stream);

/* ldk_linear on a bf16 matrix in the form the engine uses for the rows of long prefill chunks (rows that reach
 * later tokens only through cached keys and values; the paper's section 4.1 fixes no precision): where more than 64
 * rows run on the big-tile matrix-core kernel, the activations enter the product rounded to fp16 (11 significant
 * bits) in one term instead of the two bf16 terms (16 bits), and the bf16 matrix entries are widened to fp16 on the
 * way to the matrix cores, which is exact for 2^-14 <= |w| <= 65504.  Other row counts and shapes, and products with
 * an operand of 4 GiB or more: exactly ldk_linear.  overflow (device memory, 4 bytes, the caller clears it) is set to 1 when the matrix or an
 * activation holds a value beyond +-65504 or not a number; y is then not to be used (the engine repeats such a
 * pass with ldk_linear's arithmetic).  scratch: ldk_linear_scratch_bytes(...) bytes.
 * W_f16 (device memory, may be NULL): the matrix as fp16, same layout as W, written by ldk_weights_to_f16 with its
 * overflow flag left clear.  The rows that take the fp16 form then read it in W's place and widen nothing on the
 * way (the other rows, e.g. those past a multiple of 256, still read W); the matrix is not looked at again.  The
 * products are those of the values W holds either way: y is bit-equal with and without the image. */
ld_status ldk_linear_f16(const void *W, const void *W_f16, const float *x, const float *g, float eps, int32_t T,
                         int32_t N, int32_t K, int32_t epilogue, float *y, void *scratch, size_t scratch_bytes,
                         int32_t *overflow, void *stream);

/* out[i] = W[i] as fp16 for the n entries of a bf16 matrix (n a multiple of 8; both device memory, out n * 2
 * bytes, not overlapping W): exact for 2^-14 <= |w| <= 65504, smaller magnitudes lose their low bits (truncated
 * toward zero).  overflow (device memory, 4 bytes, the caller clears it) is set to 1 when an entry lies beyond
 * +-65504 or is not a number; the image is then not to be used.  The engine keeps such
 * images where its caller attaches a buffer for them (ld_model_attach_f16_image). */
ld_status ldk_weights_to_f16(const void *W, int64_t n, void *out, int32_t *overflow, void *stream);

/* cos_sin[t, i] = (cos, sin)(pos[t] * rope_base^(-2i/hd)) for i < hd/2, as float32 pairs; the
 * angle is formed in float64 so that large positions lose no accuracy.  hd is 64 or 128. */
ld_status ldk_rope_table(const int32_t *pos, int32_t T, int32_t hd, float rope_base, float *cos_sin, void *stream);

/* Rotary embedding + cache append for T rows of a fused projection qkv [T, (H + 2 Hkv) hd]:
 * rotates every q head and k head of row t in place by the angles in cos_sin[t] (pair i =
 * elements (i, i + hd/2) of a head), then stores k and v, rounded to `dtype` (nearest even), into
 * block b = table[seq_slot[t] * table_stride + pos[t] / 16], slot s = pos[t] % 16 of pool_layer:
 *   pool_layer[b][0][kv_head][s][:] = k,     pool_layer[b][1][kv_head][:][s] = v   (values transposed).
 * pool_layer is one layer's slice of the pool: keys [block][0][Hkv][16][hd], values [block][1][Hkv][hd][16].
 * Rows of one call must address distinct (sequence, position) pairs. */
ld_status ldk_rope_kv_write(float *qkv, const float *cos_sin, const int32_t *pos, const int32_t *seq_slot,
                            const int32_t *table, int32_t table_stride, void *pool_layer, int32_t dtype, int32_t T,
                            int32_t H, int32_t Hkv, int32_t hd, void *stream);

/* Fused projection + rotary embedding + cache append: qkv[t, :] = W rmsnorm(x[t, :]; g, eps) with
 * W [(H + 2 Hkv) hd, K] (g == NULL: no normalisation), then exactly what ldk_rope_kv_write does.
 * On return the q part of qkv (first H hd floats of each row) is rotated; the k and v parts of qkv
 * are unspecified (their values are in the pool).  x [T, K], qkv [T, (H + 2 Hkv) hd]. */
ld_status ldk_qkv_rope(const void *W, int32_t dtype, const float *x, const float *g, float eps, float *qkv,
                       const float *cos_sin, const int32_t *pos, const int32_t *seq_slot, const int32_t *table,
                       int32_t table_stride, void *pool_layer, int32_t T, int32_t K, int32_t H, int32_t Hkv, int32_t hd,
                       void *scratch, size_t scratch_bytes, void *stream);

/* Scratch bytes ldk_paged_attention needs for T rows with contexts up to max_ctx (same H, Hkv, window
 * as the call). */
size_t ldk_attention_scratch_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t max_ctx, int32_t window);

/* Paged attention of T single-token queries (section 2.1): row t, head h attends to cached
 * positions 0 .. ctx_len[t]-1 of the sequence whose block-table row is seq_slot[t]:
 *   s_j = q.k_j / sqrt(hd),  p = softmax(s),  out = sum_j p_j v_j.
 * q row t, head h starts at q + t * q_stride + h * hd; out is dense [T, H, hd].
 * Query head h reads KV head h / (H / Hkv); the H / Hkv query heads of a KV head are served by one
 * workgroup (keys and values loaded once) when that ratio is 2, 4 or 8.
 * window > 0: banded attention, the row (at position ctx_len[t]-1) sees only positions
 * max(0, ctx_len[t] - window) .. ctx_len[t]-1; window == 0: every cached position.
 * ctx_len[t] >= 1.  max_ctx >= max_t ctx_len[t] sizes the launch (HOST value). */
ld_status ldk_paged_attention(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype,
                              const int32_t *table, int32_t table_stride, const int32_t *seq_slot,
                              const int32_t *ctx_len, int32_t max_ctx, int32_t T, int32_t H, int32_t Hkv,
                              int32_t hd, int32_t window, float *out, void *scratch, size_t scratch_bytes,
                              void *stream);

/* ldk_paged_attention for callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation): same arguments, same kernels and the same results,
 * without the scratch pair.  The chunk partials go to a device array built into the library, of
 * LDK_STATIC_SCRATCH_BYTES bytes, which every GPU the library is used on holds from the first call on that GPU
 * until the process ends; its address is looked up once per device.  The call allocates and frees nothing.
 * A launch whose partials (T * H * chunks * (hd + 2) floats; chunks as the launch itself is cut, at most
 * ceil(max_ctx / 64)) would not fit is refused with LD_E_RANGE before anything is launched: 64 MiB serves
 * e.g. 64 rows x 40 heads at contexts up to 16384 (42 MB).  Nothing in the array has to start at zero (every partial
 * a merge reads was written by the same call), but all calls on one GPU share it: calls that overlap on one
 * GPU (different streams, or different threads) race; calls on one stream do not. */
#define LDK_STATIC_SCRATCH_BYTES (64u << 20)
size_t ldk_static_scratch_bytes(void);
ld_status ldk_paged_attention_static(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype,
                                     const int32_t *table, int32_t table_stride, const int32_t *seq_slot,
                                     const int32_t *ctx_len, int32_t max_ctx, int32_t T, int32_t H, int32_t Hkv,
                                     int32_t hd, int32_t window, float *out, void *stream);

/* Attention for prefill segments (section 2.1: all tokens of a prompt go through the model in one
 * iteration): a segment is a run of rows of one sequence at consecutive positions whose keys
 * and values are already in the pool; row r at position p attends to cached positions 0 .. p
 * (window > 0: positions max(0, p - window + 1) .. p).
 * tiles: DEVICE int32[n_tiles][4] = (first row, number of rows (1..128), position of the first row,
 * block-table row of the sequence); a segment longer than 128 rows is given as several tiles.
 * q and out as in ldk_paged_attention.  Supported: dtype LD_BF16 with hd = 128 (LD_E_INVAL otherwise;
 * such shapes run their prefill rows through ldk_paged_attention with ctx_len = position + 1).
 * max_pos (HOST value) >= the position of every row.  When few tiles face a long context the KV range of
 * a tile is split over several workgroups whose partial results go through scratch (DEVICE, up to
 * ldk_prefill_attention_scratch_bytes() bytes are used) and are merged in split order; scratch == NULL or a
 * smaller buffer only limits the split, never the result. */
size_t ldk_prefill_attention_scratch_bytes(void);
ld_status ldk_prefill_attention(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype,
                                const int32_t *table, int32_t table_stride, const int32_t *tiles, int32_t n_tiles,
                                int32_t H, int32_t Hkv, int32_t hd, int32_t window, int32_t max_pos, float *out,
                                void *scratch, size_t scratch_bytes, void *stream);

/* ldk_prefill_attention in the form the engine uses in passes of 512 rows or more (see ldk_linear_f16): with
 * overflow != NULL the queries and the probabilities enter the matrix-core products as one fp16 term (11 significant
 * bits; two bf16 terms otherwise) and the cached keys and values are widened from bf16 to fp16, which is exact within
 * +-65504.  *overflow (DEVICE, 4 bytes, cleared by the caller) is set to 1 when a scaled query, a key or a value of a
 * position the walk touches lies beyond that range or is not a number; out is then not to be used.  overflow == NULL:
 * exactly ldk_prefill_attention. */
ld_status ldk_prefill_attention_f16(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype,
                                    const int32_t *table, int32_t table_stride, const int32_t *tiles,
                                    int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t window,
                                    int32_t max_pos, float *out, void *scratch, size_t scratch_bytes,
                                    int32_t *overflow, void *stream);

/* out[r] = smallest index of the maximum of logits[r, 0..V). */
ld_status ldk_argmax(const float *logits, int32_t R, int32_t V, int32_t *out, void *stream);

/* Token choice with temperature (section 4.1 decodes at temperature 0 = ldk_argmax; this is the same
 * decision with noise): out[r] = smallest index of the maximum of logits[r, i] / temperature[r] + g(r, i),
 * g = -log(-log(u)) standard Gumbel noise, which draws i with probability softmax(logits[r] / temperature[r]).
 * u = (k + 1/2) / 2^23 with k the top 23 bits of the SplitMix64 output function applied to
 * seed[r] + (pos[r] * V + i + 1) * 0x9E3779B97F4A7C15: a pure function of (seed, pos, i).  Rows with
 * temperature[r] == 0 are the plain argmax.  temperature, seed, pos: DEVICE arrays of R entries. */
ld_status ldk_sample(const float *logits, int32_t R, int32_t V, const float *temperature, const uint64_t *seed,
                     const int32_t *pos, int32_t *out, void *stream);

/* ---- A decode step that reads few bytes: 4-bit weights, attention over selected cache blocks, choice under rules. ---- */

/* 4-bit weights with group scales: W[n, k] = (c[n, k] - z[n, k / group]) * s[n, k / group], codes c in 0..15, group 32,
 * 64 or 128 input columns, scales s of scale_dtype (LD_F32 | LD_BF16), zero points z in 0..15 or, without them
 * (zeros NULL / 0), z = 8 everywhere.  Any N from 1 to 1048560 and K >= 1; a last group may be short.
 * ldk_linear_w4 reads a matrix from an image that is laid out once: `parts` matrices of N rows each (1; 2 for
 * LDK_SWIGLU: the gate rows, then the up rows), ldk_w4_image_bytes(...) bytes of DEVICE memory, 16-byte aligned.
 * ldk_w4_image_bytes returns 0 for arguments that no image has.
 * ldk_w4_pack lays out given codes: codes [parts * N][(K + 1) / 2] bytes, the even column in the low four bits, scales
 * and zeros [parts * N][ceil(K / group)].
 * ldk_w4_quantize rounds a matrix [parts * N, K] (dtype LD_F32 | LD_BF16, finite) to nearest: without zero points
 * s = max |w| / 7 over the group, with them s = (max - min) / 15 over the group and 0, z = round(-min / s); s is
 * rounded to scale_dtype before the codes are formed. */
size_t ldk_w4_image_bytes(int32_t N, int32_t K, int32_t group, int32_t parts, int32_t scale_dtype, int32_t zeros);
ld_status ldk_w4_pack(const uint8_t *codes, const void *scales, int32_t scale_dtype, const uint8_t *zeros, int32_t N, int32_t K,
                      int32_t group, int32_t parts, void *image, size_t image_bytes, void *stream);
ld_status ldk_w4_quantize(const void *W, int32_t dtype, int32_t N, int32_t K, int32_t group, int32_t parts, int32_t scale_dtype,
                          int32_t zeros, void *image, size_t image_bytes, void *stream);

/* ldk_linear on such an image (same epilogues, same optional RMS normalisation of the input; the image's parts follow
 * from the epilogue).  x [T, K], y [T, N] dense row-major float32, which do not overlap.  The codes are exact in the products; the
 * activations enter as two fp16 terms under a power of two of the row, sums are float32.  Of an activation at most 2^-22 of the largest of its
 * 128 columns (128 j .. + 128) gets lost, 2^-25 where it is below a quarter of that, in either case no more than 2^-11 of itself; on top of it up to
 * 2^-35 of the row's largest.  So columns beside one 2^12 and more times as large keep 11 bits of their own; where the large one's weight is zero (its
 * code the zero point), nothing of it enters and the result shows that.
 * A row of x that holds a NaN or an infinity (after the normalisation) gives NaN in all of its outputs; no other row is touched by it.
 * scratch: ldk_linear_w4_scratch_bytes(T, N, K, epilogue) bytes, 16-byte aligned, needed at every T (up to 2^20); a buffer for more rows serves fewer. */
size_t ldk_linear_w4_scratch_bytes(int32_t T, int32_t N, int32_t K, int32_t epilogue);
ld_status ldk_linear_w4(const void *image, int32_t scale_dtype, int32_t zeros, int32_t group, const float *x, const float *g, float eps,
                        int32_t T, int32_t N, int32_t K, int32_t epilogue, float *y, void *scratch, size_t scratch_bytes, void *stream);

/* 8-bit bounds of the keys of cache blocks, which ldk_sparse_attention scores with.  For physical block b and KV head j, over
 * the block's cached positions: unit[b][j] = 2^e, e = floor(log2 max |k|) - 6 (at least -126; 1 for keys that are all zero),
 *   bounds[b][j][0][i] = min(127, ceil(max_p k[p][i] / unit)),  bounds[b][j][1][i] = max(-127, floor(min_p k[p][i] / unit)).
 * A block with a key that is not finite gets unit = infinity and is always preferred by the selection.
 * bounds: int8 [n_blocks][Hkv][2][hd] (16-byte aligned), unit: float [n_blocks][Hkv], DEVICE, one pair per layer.
 * To be called after keys have been written (ldk_rope_kv_write, ldk_qkv_rope): ranges DEVICE int32 [n_ranges][3] =
 * (block-table row, first new position, end of the sequence's positions); every block that first .. end - 1 touch is described anew, over its
 * positions below end.  max_len (HOST) >= end - first of every range.  Ranges of one call name distinct blocks.  Blocks the
 * table does not map (< 0) are skipped. */
ld_status ldk_kv_summary(const void *pool_layer, int32_t dtype, const int32_t *table, int32_t table_stride, const int32_t *ranges,
                         int32_t n_ranges, int32_t max_len, int32_t Hkv, int32_t hd, int8_t *bounds, float *unit, void *stream);

/* ldk_paged_attention over `budget` of the visible blocks for each row and KV head (all of them where there are no more):
 * the first keep_first and the last keep_last (>= 1) visible blocks, and the others by descending score, the lower
 * index first among equal scores.  With q'_h the query head rounded to integers of v_h = 2^(floor(log2 max |q_h|) - 6),
 * clamped to +-127,
 *   score(b) = max over the KV head's query heads of v_h unit[b] sum_i (q'_i >= 0 ? q'_i bounds[b][0][i] : q'_i bounds[b][1][i]).
 * Sums of integers and powers of two, rounded once, to float32 (beyond its range: an infinity): the choice depends on nothing but the row and the
 * bounds (which every visible block must have).  A query head with a NaN or an infinity scores 0 everywhere.
 * out [T, H, hd]: softmax attention over the selected blocks' visible positions, arguments as in
 * ldk_paged_attention; ctx_len[t] may be 0: the row's out is 0 and it selects nothing.  max_ctx (HOST) >= every ctx_len.
 * sel (DEVICE, int32 [T, Hkv, budget]): the selected logical blocks, ascending, then -1.
 * scratch: ldk_sparse_attention_scratch_bytes(...) bytes, 16-byte aligned; a buffer for more rows or longer contexts serves less. */
size_t ldk_sparse_attention_scratch_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t max_ctx, int32_t window, int32_t budget);
ld_status ldk_sparse_attention(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype, const int8_t *bounds, const float *unit,
                               const int32_t *table, int32_t table_stride, const int32_t *seq_slot, const int32_t *ctx_len, int32_t max_ctx,
                               int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t window, int32_t budget, int32_t keep_first,
                               int32_t keep_last, float *out, int32_t *sel, void *scratch, size_t scratch_bytes, void *stream);

/* What ldk_choose applies to the logits of row r, in this order.  All pointers DEVICE; a NULL member leaves its rule out.
 *   history [R][history_stride], history_len [R], penalties [R][3] = (repetition > 0, presence, frequency):
 *     for a token i among history[r][0 .. history_len[r]), l = l > 0 ? l / repetition : l * repetition, and with c = its number among
 *     history[r][n_prompt[r] .. history_len[r]) (n_prompt NULL: 0), l -= frequency * c + (c > 0 ? presence : 0).  Tokens outside 0 .. V-1
 *     are ignored.
 *   bias_start [R + 1], bias_token, bias: l += bias[j], j the last of bias_start[r] .. bias_start[r + 1] - 1 with bias_token[j] = i.
 *   mask [mask_rows][ceil(V / 32)], mask_row [R] (NULL: row r's mask is row r): bit i % 32 of word i / 32 clear: l = -infinity.  mask_row[r] < 0:
 *     no mask; mask_row[r] >= mask_rows: no token is allowed. */
typedef struct {
    const int32_t *history, *history_len, *n_prompt;
    const float *penalties;
    const int32_t *bias_start, *bias_token;
    const float *bias;
    const uint32_t *mask;
    const int32_t *mask_row;
    int32_t history_stride, mask_rows;
} ld_token_rules;

/* Token choice under rules (HOST struct, may be NULL): token[r] = lowest index of the largest adjusted logit or, where temperature[r] > 0, the
 * draw that ldk_sample makes from the adjusted logits (temperature NULL: greedy; seed and pos as there); -1 where every
 * adjusted logit is -infinity or NaN.  adjusted (may be NULL, may be logits itself): the adjusted logits [R, V].
 * scratch: ldk_choose_scratch_bytes(R, V) bytes, 8-byte aligned.  R up to 65535, V up to 2^30. */
size_t ldk_choose_scratch_bytes(int32_t R, int32_t V);
ld_status ldk_choose(const float *logits, int32_t R, int32_t V, const ld_token_rules *rules, const float *temperature, const uint64_t *seed,
                     const int32_t *pos, float *adjusted, int32_t *token, void *scratch, size_t scratch_bytes, void *stream);

/* ---- An 8-bit paged cache, and the attention that reads it. ---- */

/* One layer's 8-bit pool.  The vector x[0 .. hd) of one position and KV head, a key or a value, stands as c[i] 2^e:
 *   e = max(floor(log2 max |x|) - 6, -126) (-126 for a zero vector),  c[i] = x[i] 2^-e rounded to nearest, ties to even, within +-127.
 * A vector with a NaN or an infinity (or beyond the range of float32) has e = -128, c = 0 and stands for NaN in every entry.
 *   codes int8 [block][0][Hkv][16][hd] keys, [block][1][Hkv][hd][16] values (transposed, as in ldk_rope_kv_write's pool), 16-byte aligned;
 *   expo  int8 [block][2][Hkv][16] (keys, values), 16-byte aligned.
 * c 2^e is exact in bf16 and float32, so positions that go through a bf16 pool and back keep their codes.  What unwritten slots hold never
 * reaches a result.  Tables, slots and positions as in ldk_rope_kv_write; hd is 64 or 128, H a multiple of Hkv.  In every call of this
 * section blocks that a table does not map (entry < 0, or positions beyond table_stride blocks) are not touched: nothing is written to them, and no
 * position of theirs is visible.  Nothing in scratch has to be clear; calls that may overlap (on two streams) have scratch of their own. */

/* ldk_rope_table for any even rot >= 2 (the rotated part of a head; pairs i < rot / 2) and scaled frequencies: with f = rope_base^(-2i/rot),
 *   r = original f / 2 pi (turns over the original context),  g = clamp((r - low) / (high - low), 0, 1),  f' = f ((1 - g) / factor + g),
 *   cos_sin[t, i] = attention * (cos, sin)(pos[t] f'), float64 rounded once.
 * original == 0: g = 0 (all frequencies divided by factor; low and high are not looked at).  scaling (HOST) NULL: f' = f, attention 1. */
typedef struct {
    float factor;      /* > 0 */
    float low, high;   /* turns below which a frequency is divided by factor, above which it is kept; high > low */
    int32_t original;  /* context length the model was trained on, >= 0 */
    float attention;   /* on cos and sin, finite */
} ld_rope_scaling;
ld_status ldk_rope_table_scaled(const int32_t *pos, int32_t T, int32_t rot, float rope_base, const ld_rope_scaling *scaling, float *cos_sin,
                                void *stream);

/* ldk_rope_kv_write into an 8-bit pool, with the norms of q and k heads in the same pass.  Row t of qkv starts at qkv + t * qkv_stride (H q heads, Hkv k
 * heads, Hkv v heads of hd floats).  With q_gain [hd]: every q head x becomes x / sqrt(mean x^2 + eps) * q_gain; k_gain likewise (NULL: none).
 * Then the first rot (even, 0 .. hd) elements of q and k heads are rotated by cos_sin [T, rot / 2]: pair i = elements (i, i + rot / 2), or with
 * interleaved != 0 (2i, 2i + 1).  q goes to q_out + t * q_out_stride [H hd]; q_out may be qkv itself with the same stride, otherwise they do not
 * overlap.  k and v go into the pool.  Norms, rotation and codes are computed in float64, in an order that does not depend on T: a row gets the same codes in
 * any call.  A row with
 * pos[t] < 0 is padding: nothing of it is written.  Rows of one call address distinct (sequence, position) pairs. */
ld_status ldk_rope_kv_write_q8(const float *qkv, int32_t qkv_stride, const float *q_gain, const float *k_gain, float eps, const float *cos_sin,
                               int32_t rot, int32_t interleaved, const int32_t *pos, const int32_t *seq_slot, const int32_t *table,
                               int32_t table_stride, int8_t *codes, int8_t *expo, int32_t T, int32_t H, int32_t Hkv, int32_t hd, float *q_out,
                               int32_t q_out_stride, void *stream);

/* Cached positions from a pool of the model's type (one layer, as ldk_rope_kv_write leaves it) into an 8-bit one, and back: a sequence that
 * waits can be set aside at half its size.  ranges DEVICE int32 [n_ranges][3] = (block-table row, the same in both tables; first position; end):
 * positions first .. end - 1 of row table of the source go to the same positions of the destination's table; nothing else is written.  max_len (HOST) >=
 * end - first of every range, positions beyond it stay behind.  Ranges of one call name distinct positions. */
ld_status ldk_kv_to_q8(const void *pool_layer, int32_t dtype, const int32_t *table, int32_t table_stride, int8_t *codes, int8_t *expo,
                       const int32_t *q8_table, int32_t q8_table_stride, const int32_t *ranges, int32_t n_ranges, int32_t max_len, int32_t Hkv,
                       int32_t hd, void *stream);
ld_status ldk_kv_from_q8(const int8_t *codes, const int8_t *expo, const int32_t *q8_table, int32_t q8_table_stride, void *pool_layer, int32_t dtype,
                         const int32_t *table, int32_t table_stride, const int32_t *ranges, int32_t n_ranges, int32_t max_len, int32_t Hkv,
                         int32_t hd, void *stream);

/* ldk_paged_attention over an 8-bit pool.  Row t, at position p = ctx_len[t] - 1, sees positions max(first[t], ctx_len[t] - window) .. p of its
 * sequence (first NULL: 0; window 0: no band); ctx_len[t] may be 0, and a row that sees nothing gives 0.
 *   s_j = q.k_j / sqrt(hd);  softcap > 0 (1e-30 at least): s_j = softcap tanh(s_j / softcap);  slopes (DEVICE [H], may be NULL): s_j += slopes[h] (j - p);
 *   out = sum_j softmax(s)_j v_j.
 * A query enters as a multiple of 1 / 8355711 of its largest entry, a weight times its value's 2^e with 22 bits, of which at most 2^-38 of the row's largest such product
 * gets lost besides, and a weight below 2^-126 of the row's largest counts as 0; codes are exact, sums float32.  Range: scores below 2^126 in magnitude.  A query head with a NaN or an infinity gives NaN, as does a head that sees a key or value that stands for NaN.  max_ctx (HOST) >= every ctx_len.
 * scratch: ldk_attention_q8_scratch_bytes(...) bytes, 16-byte aligned; a buffer for more rows or longer contexts serves less. */
size_t ldk_attention_q8_scratch_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t max_ctx, int32_t window);
ld_status ldk_paged_attention_q8(const float *q, int32_t q_stride, const int8_t *codes, const int8_t *expo, const int32_t *table,
                                 int32_t table_stride, const int32_t *seq_slot, const int32_t *first, const int32_t *ctx_len, int32_t max_ctx,
                                 int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t window, float softcap, const float *slopes, float *out,
                                 void *scratch, size_t scratch_bytes, void *stream);

/* ldk_prefill_attention over an 8-bit pool.  tiles: DEVICE int32 [n_tiles][6] = (first row, number of rows 1 .. 128, position of the first row,
 * block-table row, first visible position, prefix length).  The row at position p sees positions max(first visible, p - window + 1) ..
 * max(p, prefix - 1): a band (window 0: none), a document's start and a prefix that sees all of itself; a row that sees nothing gives 0.
 * Scores as in ldk_paged_attention_q8.  Rows that no tile names are left as they are.  max_pos (HOST) >= every max(p, prefix - 1).
 * Range: keys below 2^120, scores below 2^126 in magnitude; values that a tile sees within a factor of 2^85 of each other, or of 1 where 64 of them in a row are zero; values
 * below 2^-119 count as zero.  Where a row's weight lies all but 2^-20 on zero values, or on values so much smaller than others, weights have 18 bits, and what gets lost besides
 * is at most 2^-120 of the largest 2^e.
 * scratch: ldk_prefill_attention_q8_scratch_bytes(...) bytes, 16-byte aligned; a buffer for more tiles or longer contexts serves less. */
size_t ldk_prefill_attention_q8_scratch_bytes(int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t max_pos, int32_t window);
ld_status ldk_prefill_attention_q8(const float *q, int32_t q_stride, const int8_t *codes, const int8_t *expo, const int32_t *table,
                                   int32_t table_stride, const int32_t *tiles, int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t window,
                                   float softcap, const float *slopes, int32_t max_pos, float *out, void *scratch, size_t scratch_bytes,
                                   void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LD_KERNELS_H */
