/*
 * d2c_q8.h -- the 8-bit operators beside the d2Cache step library (include/d2c.h): a K/V cache held in 8 bits
 * with a scale for each block of 64 rows and kv head, the attention that reads it, products in 8-bit integers
 * with scales per token and channel, and the eviction of cache rows by the attention weight they drew.
 *
 * Conventions are those of d2c.h (0 or a negative error code, never throws; on an argument error nothing has been
 * launched or written; device pointers unless marked (host); all work asynchronous on `stream`), and
 *   - a d2c_q8 handle holds the geometry and the workspace and no weights; it belongs to the device that is current
 *     at d2c_q8_init, and calls with another device current are refused (D2C_EINVAL);
 *   - no call but d2c_q8_init allocates, copies to the host or waits, so each can be captured into a HIP graph;
 *   - a handle is not thread-safe, and calls (or replays of graphs captured from calls) that share a handle must not
 *     overlap in time: they share its workspace.  d2c_q8_update, _read, _weigh, _evict and _pack use no workspace;
 *   - what a call writes must not overlap what it reads (but the caches that it refreshes, which it may read for other
 *     sequences) or other outputs: refused with D2C_EINVAL, as far as the call's own sizes tell;
 *   - T is float (D2C_F32) or bfloat16 (D2C_BF16), as the handle's dtype says: queries, K/V rows, outputs, activations
 *     and the weights given to d2c_q8_pack;
 *   - pointers to T and to codes are multiples of 16 bytes, others of their element's size (D2C_EINVAL).
 *
 * How values become codes.  scale(a) = fl32(a / 127) of the largest magnitude a, and 0 where a < 2^-100.
 * code(x, s) = the whole number in [-127, 127] nearest to the real quotient x / s, ties to even; 0 where s = 0.
 *
 * The cache of n rows has ceil(n / 64) blocks, each n_kv_heads * 64 * head_dim bytes of K and as many of V; the last
 * block is whole even if n is not a multiple of 64.  It starts as bytes of 128 and scales of 0 (every value 0), or with an
 * update of all its rows.  A byte is its code + 128.  With block b, kv head h, row t of the
 * block and dimension d (D = head_dim), base = (b * n_kv_heads + h) * 64 * D:
 *   K at base + (d / 16) * 1024 + t * 16 + d % 16          V at base + (t / 4) * 4 * D + d * 4 + t % 4
 *   scales at b * n_kv_heads + h.  value = code * scale.
 */
#ifndef D2C_Q8_H
#define D2C_Q8_H

#include <stdint.h>

#include "d2c.h"

#ifdef __cplusplus
extern "C" {
#endif

#define D2C_Q8_BLOCK 64   /* cache rows that share a scale */

typedef struct d2c_q8 d2c_q8;   /* opaque; created by d2c_q8_init, freed by d2c_q8_destroy */

typedef struct {
  int32_t n_heads, n_kv_heads, head_dim;   /* head_dim 64 or 128; n_heads a multiple of n_kv_heads */
  int32_t dtype;       /* D2C_F32 or D2C_BF16                                                      */
  int32_t max_seq;     /* largest L of a cache, up to 2^24; 0 = the cache calls are not used       */
  int32_t max_rows;    /* query rows of one d2c_q8_attention call, summed over its sequences, or
                          rows of one d2c_q8_linear call; up to 2^16                               */
  int32_t max_batch;   /* sequences of one call, up to 256; 0 = 1                                  */
  int32_t max_k;       /* largest contraction of d2c_q8_linear, up to 2^16; 0 = it is not used     */
  int32_t max_n;       /* largest N of d2c_q8_linear, up to 2^20; 0 = it is not used               */
} d2c_q8_dims;

/* Codes and scales of one layer's cache, caller-owned; sizes as above. */
typedef struct {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float*   k_scale;
  float*   v_scale;
} d2c_q8_cache;

/* One sequence of a call.  idx is NULL for the rows L - m .. L - 1 (a filled or continued cache). */
typedef struct {
  d2c_q8_cache cache;    /* at least L rows                                                     */
  const int32_t* idx;    /* [m] positions in [0, L) of new_k / new_v, ascending, distinct       */
  const void* new_k;     /* T [m, d_kv] refreshed rows, or NULL (both) to leave the cache as is */
  const void* new_v;
  const void* q;         /* T [m, d_q]                                    (d2c_q8_attention)    */
  void*  out;            /* T [m, d_q]                                    (d2c_q8_attention)    */
  float* attn_avg;       /* [m, L] mean over the heads of the softmax rows, or NULL (as above);
                            a call's averages have fewer than 2^23 tiles of 32 rows x 64 keys   */
  int32_t m, L;          /* (host) m = 0 is legal and leaves the sequence alone                 */
} d2c_q8_seq;

int d2c_q8_init(const d2c_q8_dims* dims, d2c_q8** out);
int d2c_q8_destroy(d2c_q8* ctx);
/* Text of the last error of this handle (ctx NULL: of this thread's last d2c_q8_init that failed). */
const char* d2c_q8_last_error(const d2c_q8* ctx);
/* Bytes of device workspace the handle holds. */
int64_t d2c_q8_workspace_bytes(const d2c_q8* ctx);

/* Sizes of a cache of `rows` rows: bytes of K codes (V: as many) and floats of K scales (V: as many). */
int d2c_q8_cache_size(const d2c_q8* ctx, int64_t rows, int64_t* code_bytes, int64_t* scale_floats);

/* Refreshed rows go into the caches: row r of new_k / new_v becomes row idx[r].  A block all of whose rows below L are
 * refreshed gets the scale of its new rows.  In other blocks the scale stays where the new rows fit; where they do not, it
 * becomes max(scale(new rows), 1.25 * old scale) and the other rows' codes become code(code * old, new) -- at least a quarter
 * at a time, so that many small growths cannot let a value drift away with its scale.  A value that is not finite counts
 * for no scale: NaN is stored as 0, an infinity as the largest code of its sign.  Indices outside [0, L) are left out;
 * indices that are not ascending and distinct leave the blocks of 64 rows that they name undefined, and nothing else.  L is
 * the cache's length: rows from L on of the block that holds row L - 1 have no defined values once that block is refreshed.
 * Two sequences of a call must not refresh the same cache (D2C_EINVAL). */
int d2c_q8_update(d2c_q8* ctx, const d2c_q8_seq* seqs, int32_t batch, void* stream);

/* d2c_q8_update of the sequences that give new_k / new_v, then attention of each sequence's m query rows against all L rows
 * of its cache, no mask; sequences may share a cache that at most one of them refreshes.  Scores, softmax and sums are fp32;
 * scores (q k^T / sqrt(D)) are meant to stay within 2^22, and L times the values of V within 2^112: beyond, a row can turn NaN
 * or infinite.
 * q enters as fp16 pieces of a row scaled by a power of two, one for bf16 (exact down to 2^-32 of the row's largest
 * magnitude, to the nearest 2^-39 of it below), two for float (within 2^-23, or 2^-39 of the largest).  Probabilities are
 * rounded to 11 bits for bf16 and 22 for float, those below 2^-25 (float: 2^-18) of a row's largest to the nearest 2^-35
 * (2^-39) of it. */
int d2c_q8_attention(d2c_q8* ctx, const d2c_q8_seq* seqs, int32_t batch, void* stream);

/* Values of cache rows: out_k / out_v T [n, d_kv] (either may be NULL) = rows idx[0 .. n) of the cache of L rows, or rows
 * 0 .. n - 1 where idx is NULL; n up to 2^24.  An index outside [0, L) gives zeros. */
int d2c_q8_read(d2c_q8* ctx, const d2c_q8_cache* cache, int32_t L, const int32_t* idx, int32_t n,
                void* out_k, void* out_v, void* stream);

/* Weights for d2c_q8_linear: w T [N, K] -> codes (d2c_q8_weight_bytes(N, K) bytes, laid out for the matrix cores) and a
 * scale for each of the N channels.  K must be a multiple of 16 bytes of T.  w is not needed afterwards. */
int64_t d2c_q8_weight_bytes(int32_t N, int32_t K);
int d2c_q8_pack(d2c_q8* ctx, const void* w, int32_t N, int32_t K, int8_t* codes, float* scale, void* stream);

/* out[m, N] (float) = a[m, K] w[N, K]^T with each row of a quantised to 8 bits by its own largest magnitude: the sums are
 * exact whole numbers, made float, times the row's scale, times the channel's.  A row of a, or a channel of w, that holds a NaN or an
 * infinity gives NaN in its outputs and in no others. */
int d2c_q8_linear(d2c_q8* ctx, const void* a, int32_t m, const int8_t* codes, const float* scale, int32_t N, int32_t K,
                  float* out, void* stream);

/* Accumulated attention: weight[j] += sum_r floor(clamp(attn_avg[r, j], 0, 1) * 2^32) for j < L (NaN counts as 0).
 * attn_avg: float [m, L], as the attention calls leave it, m and L up to 2^24; the sums hold 2^31 such rows.  Whole numbers:
 * the order of the sum does not matter. */
int d2c_q8_weigh(d2c_q8* ctx, const float* attn_avg, int32_t m, int32_t L, int64_t* weight, void* stream);

/* Keeps n_keep of the L rows of a cache: those of largest weight (negative ones count as 0), ties to the lowest index; rows
 * with protect[j] != 0 (protect may be NULL) come before all others.  kept [n_keep] out: their positions, ascending.
 * Row i of dst is row kept[i] of src: a block of dst has the largest scale its rows had, codes of rows with another scale
 * become code(code * old, new).  kept_weight [n_keep] out (may be NULL): weight[kept], negative ones as 0.  dst holds
 * ceil(n_keep / 64) blocks and must not overlap src. */
int d2c_q8_evict(d2c_q8* ctx, const d2c_q8_cache* src, int32_t L, const int64_t* weight, const uint8_t* protect,
                 int32_t n_keep, const d2c_q8_cache* dst, int32_t* kept, int64_t* kept_weight, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* D2C_Q8_H */
