/*
 * libtsvd -- what a served transformer layer needs beside its ternary products (tsvd.h): the projections that
 * stay dense, in 8-bit integers, and the attention over a key/value cache held in 4 bits.
 *
 * The paper converts linear layers of BERT-base and OPT-6.7B and runs them inside those models; a layer that is
 * not converted, and the attention between two converted ones, have no counterpart in it.  These calls follow
 * tsvd.h: plain C, pointers and sizes, a status from every call, arguments checked on the host before any launch,
 * all work asynchronous on the given stream unless stated otherwise, no CPU implementation behind them.  Work runs on
 * the current device, where stream and pointers have to belong; a handle of another device is refused with TSVD_E_CUDA.
 */
#ifndef TSVD_SERVING_H
#define TSVD_SERVING_H

#include "tsvd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- 8-bit integers with a scale for each token and channel ------------------------------------------------- */

/*
 * tsvd_quantize -- 8-bit integers with one scale per row:
 *     a_b = max_n |x_bn|,   scale_b = a_b * (1 / 127),   q_bn = rint(x_bn * ((1 / a_b) * 127))
 * in fp32 (every reciprocal and product rounded to nearest, rint to even), so -127 <= q <= 127.
 *
 *   x      device, TSVD_F32 or TSVD_BF16, row b at x + b*ldx (elements, ldx >= cols)
 *   q      device, row b at q + b*ldq (ldq >= cols); bytes between cols and ldq are not written
 *   scale  device, float [rows]
 * A row whose largest magnitude is 0, or so small (below 2^-100) that 1 / a_b might overflow, becomes q = 0.
 * A row that holds a NaN or an infinity gets a scale that is not finite (and unspecified q), so that what is
 * computed from it is not finite either.  rows = 0 does nothing (and looks at no pointer).  Any alignment that the types allow; 16-byte
 * aligned rows are read 16 bytes at a time.
 * Errors: E_NULL, E_SHAPE, E_TOOBIG (cols above 2^31 - 2^16), E_DTYPE, E_ALIGN (a pointer is not a multiple of its type's size), E_CUDA.
 */
tsvd_status_t tsvd_quantize(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, int8_t* q,
                            long long ldq, float* scale, void* stream);

/* tsvd_dequantize -- y_bn = q_bn * scale_b, as TSVD_F32 or TSVD_BF16; layout and errors as tsvd_quantize. */
tsvd_status_t tsvd_dequantize(const int8_t* q, long long ldq, const float* scale, long long rows, int cols, void* y,
                              tsvd_dtype_t dtype, long long ldy, void* stream);

/*
 * tsvd_rms_norm -- root-mean-square norm of rows, the residual added on the way, the result as numbers or in 8 bits:
 *     h_bn = x_bn + residual_bn, rounded to x's type (x itself without a residual)
 *     rho_b = 1 / sqrt(mean_n h_bn^2 + eps)
 *     y:  y_bn = h_bn * rho_b * w_n, computed in fp32, rounded once to x's type
 *     q:  t_bn = h_bn * w_n,  a_b = max_n |t_bn|,  q_bn = rint(t_bn * ((1 / a_b) * 127)),  scale_b = (a_b * (1 / 127)) * rho_b
 * The sum of squares is taken in fp32, and once more in 64 bits for a row whose squares leave fp32's range.  q is
 * elementwise in fp32 from h and w (every reciprocal and product rounded to nearest, rint to even) and does not depend on rho.
 * It is what tsvd_i8_forward takes as TSVD_I8 rows with x_scale.
 *
 *   x         device, TSVD_F32 or TSVD_BF16, row b at x + b*ldx (elements, ldx >= cols)
 *   residual  device, like x, or NULL; then h is NULL too
 *   h         device, like x, receives the sum (the next layer's residual).  It may be x or the residual itself (the same
 *             pointer and row stride), otherwise it must not overlap them
 *   weight    device, [cols], TSVD_F32 or TSVD_BF16
 *   eps       1e-12 or more
 *   y         device, like x, or NULL; may be x itself, where there is no residual
 *   q, scale  device, row b at q + b*ldq (ldq >= cols), scale float [rows]; NULL where y is given.  One of the two results.
 * A row with a NaN or an infinity gets results that are not all finite (in 8 bits a scale that is not finite); with finite weights
 * no other row does, but for 8-bit rows one of whose products t leaves fp32's range: a_b, and with it scale_b, is then infinite.
 * A row whose a_b is below 2^-100 becomes q = 0.  rows = 0 does nothing.
 * Errors: E_NULL (also both results, or none), E_SHAPE, E_TOOBIG (cols above 2^31 - 2^16), E_DTYPE, E_VALUE (eps), E_ALIGN, E_CUDA.
 */
tsvd_status_t tsvd_rms_norm(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, const void* residual,
                            long long ldr, void* h, long long ldh, const void* weight, tsvd_dtype_t weight_dtype, float eps,
                            void* y, long long ldy, int8_t* q, long long ldq, float* scale, void* stream);

typedef struct tsvd_i8_s* tsvd_i8_t; /* opaque; owns device memory on one GPU */

/*
 * tsvd_i8_pack -- keep the weights of a linear layer in 8 bits:  W [M,N] row-major, one scale per output channel.
 *   W        int8, row m at W + m*ldw (ldw >= N); w_scale float [M]; bias float [M] or NULL.
 *            Host or device pointers; copied.  tsvd_quantize on the rows of a float matrix makes W and w_scale.
 *            Device sources must be ready: the copies wait for no stream of the caller's (the torch front does).
 * The copy is cut into the 128 x 128 tiles that the tensor-core kernels read.
 * Synchronous.  Errors: E_NULL, E_SHAPE, E_TOOBIG (N above TSVD_I8_MAX_N: a sum of N products of two 8-bit values
 * must fit 32 bits), E_DTYPE (flags is not 0), E_NOMEM, E_CUDA.
 */
#define TSVD_I8_MAX_N 131071
tsvd_status_t tsvd_i8_pack(const int8_t* W, long long ldw, const float* w_scale, const float* bias, int M, int N,
                           unsigned flags, tsvd_i8_t* out);

/*
 * tsvd_i8_forward -- y_bm = (sum_n q_bn W_mn) * scale_b * w_scale_m + bias_m  for B tokens.
 *
 *   x        device, row b at x + b*ldx (elements, ldx >= N).
 *            TSVD_I8: the q above, with x_scale device float [B] (NULL: all ones);
 *            TSVD_F32, TSVD_BF16: quantised inside the call exactly as tsvd_quantize does; x_scale must be NULL
 *   y        device, row b at y + b*ldy (ldy >= M): fp32 for TSVD_F32 and TSVD_I8, bf16 for TSVD_BF16;
 *            TSVD_FLAG_OUT_F32 makes it fp32, TSVD_FLAG_OUT_BF16 bf16
 *   flags    one of those two, or 0; TSVD_FLAG_TEST_STALL (tsvd.h) as well: the tokens never reach the product, its waits run
 *            out after some milliseconds, y is unspecified and tsvd_i8_last_status reports TSVD_E_TIMEOUT
 * The sum is exact (32-bit integers); it is rounded once to fp32, multiplied by scale_b and by w_scale_m, the bias
 * added in fp32, and rounded once more where y is bf16.  B = 0 does nothing.
 * Calls on one handle share its scratch and must be ordered, as with tsvd_forward; the scratch grows (with one
 * device synchronisation) on the first call with a larger B unless tsvd_i8_reserve has sized it.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_NOMEM, E_CUDA.
 */
#define TSVD_FLAG_OUT_BF16 0x2u
tsvd_status_t tsvd_i8_forward(tsvd_i8_t h, const void* x, long long ldx, const float* x_scale, void* y, long long ldy,
                              int B, tsvd_dtype_t dtype, unsigned flags, void* stream);
tsvd_status_t tsvd_i8_reserve(tsvd_i8_t h, int B_max, tsvd_dtype_t dtype);
tsvd_status_t tsvd_i8_info(tsvd_i8_t h, int* M, int* N, size_t* packed_bytes);
/* TSVD_E_TIMEOUT if a bounded device-side wait gave up since the last read (synchronise first), else TSVD_OK. */
tsvd_status_t tsvd_i8_last_status(tsvd_i8_t h);
void tsvd_i8_destroy(tsvd_i8_t h);

/* ---- low-rank adapters of many requests beside a shared projection ------------------------------------------- */

typedef struct tsvd_adapters_s* tsvd_adapters_t; /* opaque; owns device memory on one GPU */

/*
 * tsvd_adapters_create -- room for n_slots adapters of a projection from N to M numbers:  A [rank, N], B [M, rank], a factor
 * each, ranks up to max_rank (at most TSVD_ADAPTERS_MAX_RANK).  Every slot is empty at first.
 * Synchronous.  Errors: E_NULL, E_SHAPE, E_TOOBIG (also N above 2^24, M above 2^21), E_NOMEM, E_CUDA.
 */
#define TSVD_ADAPTERS_MAX_RANK 128
tsvd_status_t tsvd_adapters_create(int N, int M, int max_rank, int n_slots, tsvd_adapters_t* out);

/*
 * tsvd_adapters_set -- an adapter into a slot, in the stream's order: calls ahead on the stream use what the slot held before.
 *   A  device, row r at A + r*lda (elements, lda >= N);  B  device, row m at B + m*ldb (ldb >= rank); TSVD_F32 or TSVD_BF16.
 *      Copied, and kept in bf16: fp32 weights are rounded once here.
 *   rank = 0 empties the slot (A and B are not looked at).
 * Errors: E_NULL, E_INDEX (slot), E_SHAPE, E_DTYPE, E_ALIGN, E_CUDA.
 */
tsvd_status_t tsvd_adapters_set(tsvd_adapters_t h, int slot, const void* A, long long lda, const void* B, long long ldb,
                                tsvd_dtype_t dtype, int rank, float scale, void* stream);

/*
 * tsvd_adapters_forward -- out_i = base_i + scale_s * B_s (A_s x_i)  for n_rows rows, s = slots[sequence of row i].
 *   x         device, row i at x + i*ldx (ldx >= N): TSVD_F32, TSVD_BF16, or TSVD_I8 with x_scale device float [n_rows]
 *             (NULL: all ones), as tsvd_i8_forward takes them
 *   base      device, row i at base + i*ldb (ldb >= M), out_dtype: the shared projection's result; NULL: zeros
 *   out       device, row i at out + i*ldo (ldo >= M), TSVD_F32 or TSVD_BF16.  May be base itself (same pointer and stride)
 *   slots     device, int32 [n_seq]: the slot of each sequence; -1 or an empty slot: none, the row becomes base's.  A number
 *             below -1 or from n_slots on counts as none and makes tsvd_adapters_last_status report TSVD_E_INDEX
 *   q_start   device, int32 [n_seq + 1], ascending: the rows q_start[s] .. q_start[s+1]-1 belong to sequence s; NULL: one row each.  Rows
 *             below q_start[0] or from q_start[n_seq] on belong to none and are not written
 * Weights are bf16; sums, A x and the result's addition fp32 (see adapters.cu); one rounding of the result.  Rows and
 * adapters do not disturb each other: what is not finite in one stays there.
 * Calls on one handle share its scratch and must be ordered; it grows on the first call with more rows unless
 * tsvd_adapters_reserve has sized it (outgrown scratch lives as long as the handle: captured graphs stay valid).
 * Errors: E_NULL, E_SHAPE, E_TOOBIG (n_rows or n_seq above 2^30), E_DTYPE, E_ALIGN, E_NOMEM, E_CUDA.
 */
tsvd_status_t tsvd_adapters_forward(tsvd_adapters_t h, const void* x, long long ldx, const float* x_scale, tsvd_dtype_t dtype,
                                    const void* base, long long ldb, void* out, long long ldo, tsvd_dtype_t out_dtype,
                                    const int* slots, const int* q_start, int n_seq, int n_rows, void* stream);
/*
 * tsvd_adapters_forward_ex -- the same with flags: 0 or TSVD_FLAG_TEST_STALL (tsvd.h).  With that the weights never reach the products
 * of sequences of many rows (those on tcgen05), their waits run out after some milliseconds, out is unspecified and
 * tsvd_adapters_last_status reports TSVD_E_TIMEOUT; the other forms wait for nothing and take no notice of it.
 */
tsvd_status_t tsvd_adapters_forward_ex(tsvd_adapters_t h, const void* x, long long ldx, const float* x_scale, tsvd_dtype_t dtype,
                                       const void* base, long long ldb, void* out, long long ldo, tsvd_dtype_t out_dtype,
                                       const int* slots, const int* q_start, int n_seq, int n_rows, unsigned flags, void* stream);
/* Scratch for calls of up to rows_max rows, so that none of them allocates. */
tsvd_status_t tsvd_adapters_reserve(tsvd_adapters_t h, int rows_max);
tsvd_status_t tsvd_adapters_info(tsvd_adapters_t h, int* N, int* M, int* max_rank, int* n_slots, size_t* bytes);
/* Device status since the last read (synchronise first): TSVD_E_TIMEOUT if a bounded wait gave up (the results are then
 * unspecified), else TSVD_E_INDEX if a slot number was out of range, else TSVD_OK. */
tsvd_status_t tsvd_adapters_last_status(tsvd_adapters_t h);
void tsvd_adapters_destroy(tsvd_adapters_t h);

/* ---- keys and values in 4 bits ------------------------------------------------------------------------------- */

typedef struct tsvd_kv4_s* tsvd_kv4_t; /* opaque; owns device memory on one GPU */

/*
 * tsvd_kv4_create -- a pool of n_pages pages, each for page_tokens positions of n_kv_heads keys and values of
 * head_dim numbers.  head_dim is 64 or 128, page_tokens a multiple of 16.
 *
 * What is kept of a key or value: per position, head and group of 32 consecutive numbers
 *     step = fp16((hi - lo) * (1 / 15)),  base = fp16(lo),  code = clamp(rint((x - base) * (1 / step)), 0, 15)
 * with lo and hi the group's smallest and largest number (clamped to +-65000), arithmetic in fp32; step = 0 makes
 * code = 0.  It stands for code * step + base.  5 bits a number in all.
 *
 * Which pages belong to which sequence is the caller's business: every call below takes
 *   page_table  device, int32 [n_seq][max_pages]: page_table[s][p] holds positions p*page_tokens .. of sequence s
 *   seq_len     device, int32 [n_seq]: positions of sequence s in the cache, the call's new ones included
 *   q_start     device, int32 [n_seq + 1]: the call's rows q_start[s] .. q_start[s+1]-1 are the last positions of
 *               sequence s, in order; NULL: one row per sequence
 *   n_rows      q_start[n_seq] (n_seq where q_start is NULL); rows below q_start[0], or beyond q_start[n_seq] where n_rows
 *               is larger, belong to no sequence: they are not written (append, attend) and read as zeros (read)
 * All three are read on the device: a captured graph serves them as they change.  A page number outside the pool or a
 * sequence longer than its pages makes tsvd_kv4_last_status report TSVD_E_INDEX, and so does a row before position 0 in
 * append and read; such a position is not written (append), reads as zeros (read) and is not seen (attend).  An unused
 * slot of a batch (seq_len 0 with a row) is therefore fine in attend, which gives it zeros.
 * Calls on one handle must be ordered on one stream (or otherwise serialised).  More than 2^31 - 2^16 sequences or rows: E_TOOBIG.
 * Synchronous.  Errors: E_NULL, E_SHAPE, E_TOOBIG (n_pages * page_tokens above 2^31 - 1, page_tokens above 2^24), E_NOMEM, E_CUDA.
 */
tsvd_status_t tsvd_kv4_create(int n_kv_heads, int head_dim, int page_tokens, long long n_pages, tsvd_kv4_t* out);

/*
 * tsvd_kv4_append -- put the keys and values of n_rows new positions into the cache.
 *   k, v  device, TSVD_F32 or TSVD_BF16: head g of row i at k + i*ldk + g*head_dim (ldk >= n_kv_heads*head_dim),
 *         so that slices of one projection's output are taken as they are; v and ldv likewise.
 *         Finite; magnitudes above 65000 are clamped.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN (k or v not a multiple of its type's size), E_CUDA.
 */
tsvd_status_t tsvd_kv4_append(tsvd_kv4_t h, const void* k, long long ldk, const void* v, long long ldv, tsvd_dtype_t dtype,
                              const int* page_table, int max_pages, const int* seq_len, const int* q_start, int n_seq,
                              int n_rows, void* stream);

/*
 * tsvd_kv4_append_rotated -- tsvd_kv4_append with the rotation by position on the way: row i stands at position
 * P_i = seq_len[s] - (rows of s) + (i - q_start[s]); of every head of q and k the first `turned` numbers are rotated in pairs,
 *     (u, v)  ->  (u * cos - v * sin,  v * cos + u * sin)      every product and sum rounded to fp32
 * with cos = table[P_i * turned + p] and sin = table[P_i * turned + turned/2 + p] for pair p.  Keys then go into the cache from
 * fp32, queries are rounded once to their type; the other numbers of a head, and v, are taken as they are.
 *   q         device, like k: head a of row i at q + i*ldq + a*head_dim (ldq >= n_heads*head_dim); n_heads = 0: no queries
 *   q_out     device, like q; must not overlap q, k or v
 *   table     device, float [positions][turned], as tsvd_rotary_table makes it
 *   turned    even, 2 .. head_dim
 *   interleaved  0: pair p is the numbers (p, p + turned/2); else (2p, 2p + 1)
 * A position behind the table makes tsvd_kv4_last_status report TSVD_E_INDEX, as does one before 0 or outside the pages; its
 * keys and values are not written, and its row of q_out is zeros where the table has no such position.  Rows that belong to no
 * sequence are not written.
 * Errors: those of tsvd_kv4_append; E_VALUE (q_out is q).
 */
tsvd_status_t tsvd_kv4_append_rotated(tsvd_kv4_t h, const void* q, long long ldq, void* q_out, long long ldqo, int n_heads,
                                      const void* k, long long ldk, const void* v, long long ldv, tsvd_dtype_t dtype,
                                      const float* table, int positions, int turned, int interleaved, const int* page_table,
                                      int max_pages, const int* seq_len, const int* q_start, int n_seq, int n_rows, void* stream);

/*
 * tsvd_rotary_table -- table[P * turned + p] = amplitude * cos(P * rates[p]), and sin at + turned/2, for P = 0 .. positions-1
 * and p = 0 .. turned/2-1; angles in 64 bits, one rounding to fp32.
 *   table  device, float [positions][turned];  rates  device, double [turned/2]
 * Errors: E_NULL, E_SHAPE, E_ALIGN, E_CUDA.
 */
tsvd_status_t tsvd_rotary_table(float* table, int positions, int turned, const double* rates, float amplitude, void* stream);

/* tsvd_kv4_read -- the inverse: what the cache holds for those rows, into k and v (the numbers the codes stand for, as
 * TSVD_F32 or TSVD_BF16).  Arguments and errors as tsvd_kv4_append. */
tsvd_status_t tsvd_kv4_read(tsvd_kv4_t h, void* k, long long ldk, void* v, long long ldv, tsvd_dtype_t dtype,
                            const int* page_table, int max_pages, const int* seq_len, const int* q_start, int n_seq,
                            int n_rows, void* stream);

/*
 * tsvd_kv4_attend -- attention of n_rows queries over their sequences' cached keys and values:
 *     out_i,a = sum_j p_ij v_j,   p_ij = exp(scale * q_i,a . k_j) / sum_j' exp(scale * q_i,a . k_j')
 * query head a uses key/value head a / (n_heads / n_kv_heads); row i of sequence s stands at position
 * P_i = seq_len[s] - (rows of s) + (i - q_start[s]) and sees the positions j < seq_len[s] with
 *     j <= P_i                with TSVD_FLAG_CAUSAL
 *     j >  P_i - window       where window > 0
 * A row that sees nothing (seq_len 0, for instance) gets zeros.  Append the new keys first.
 *
 *   q, out   device, TSVD_BF16 or TSVD_F32 both: head a of row i at q + i*ldq + a*head_dim (ldq >= n_heads*head_dim);
 *            out and ldo likewise.  Rows do not disturb each other: an infinity or a NaN in a row of q spoils that row's
 *            result only.
 *   n_heads  a multiple of the cache's n_kv_heads
 *   max_q    at least the rows of any sequence; rows beyond it are not computed.  It chooses the kernel, for all sequences of
 *            the call: up to 16 rows a key/value head are far faster by the one for few rows
 *   max_kv   at least any seq_len; 0: max_pages * page_tokens.  A tighter bound spreads the work better and
 *            changes no result
 *   flags    TSVD_FLAG_CAUSAL, TSVD_FLAG_PATH_SIMPLE (CUDA-core kernel in fp32), TSVD_FLAG_TEST_STALL (bf16 on the tensor
 *            cores: the cached positions never arrive, the waits run out after some milliseconds, out is unspecified and
 *            tsvd_kv4_last_status reports TSVD_E_TIMEOUT), or several
 * bf16: products of tensor-core precision (q, keys and values as the cache holds them in bf16 or fp16, probabilities in
 * fp16), sums in fp32, one rounding of the result.  fp32: fp32 throughout.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN (q or out not 16-byte aligned, ldq or ldo not a multiple of 8 elements),
 * E_CUDA.
 */
#define TSVD_FLAG_CAUSAL 0x4u
tsvd_status_t tsvd_kv4_attend(tsvd_kv4_t h, const void* q, long long ldq, void* out, long long ldo, int n_heads,
                              tsvd_dtype_t dtype, const int* page_table, int max_pages, const int* seq_len,
                              const int* q_start, int n_seq, int n_rows, int max_q, int max_kv, float scale, int window,
                              unsigned flags, void* stream);

/*
 * tsvd_kv4_attend_sinks -- the same with the first `sinks` positions of a sequence exempt from the window: a row sees j < seq_len[s] with
 *     j <= P_i                                 with TSVD_FLAG_CAUSAL
 *     j >  P_i - window  or  j < sinks         where window > 0
 * Without a window, sinks changes nothing; sinks = 0 is tsvd_kv4_attend.  With both, pages that hold none of the positions that
 * the rows see are not looked at: they may be handed out again, their numbers in page_table be anything.
 * Errors: those of tsvd_kv4_attend; E_SHAPE (sinks below 0).
 */
tsvd_status_t tsvd_kv4_attend_sinks(tsvd_kv4_t h, const void* q, long long ldq, void* out, long long ldo, int n_heads,
                                    tsvd_dtype_t dtype, const int* page_table, int max_pages, const int* seq_len,
                                    const int* q_start, int n_seq, int n_rows, int max_q, int max_kv, float scale, int window,
                                    int sinks, unsigned flags, void* stream);

tsvd_status_t tsvd_kv4_info(tsvd_kv4_t h, int* n_kv_heads, int* head_dim, int* page_tokens, long long* n_pages,
                            size_t* pool_bytes);
/* Device status since the last read (synchronise first): TSVD_E_TIMEOUT if a bounded wait gave up, else TSVD_E_INDEX if a
 * page number or length was out of range, else TSVD_OK.  After TSVD_E_TIMEOUT the results of every tsvd_kv4_attend since the
 * read before are unspecified; this read makes the handle fit for the next one. */
tsvd_status_t tsvd_kv4_last_status(tsvd_kv4_t h);
void tsvd_kv4_destroy(tsvd_kv4_t h);

#ifdef __cplusplus
}
#endif
#endif /* TSVD_SERVING_H */
