/*
 * d2c_pg.h -- the paged K/V cache beside the d2Cache step library (include/d2c.h): rotary positions of one or several axes,
 * appending keys and values to pages with the rotation on the way, and the attention of a batch of sequences over their
 * pages, from one token each to whole prompts, causal, block-causal, windowed or without a mask.
 *
 * Conventions are those of d2c.h (0 or a negative error code, never throws; on an argument error nothing has been
 * launched or written; device pointers unless marked (host); all work asynchronous on `stream`), and
 *   - a d2c_pg handle holds the geometry, the rotation and the workspace; it belongs to the device that is current
 *     at d2c_pg_init, and calls with another device current are refused (D2C_EINVAL);
 *   - no call but d2c_pg_init allocates, copies to the host or waits, so each can be captured into a HIP graph.  Row starts,
 *     lengths, page numbers, indices and positions are read on the device: a captured call follows them as they change;
 *   - a handle is not thread-safe, and d2c_pg_attention calls (or replays of graphs captured from them) that share a handle
 *     must not overlap in time: they share its workspace.  The other calls use no workspace;
 *   - what a call writes must not overlap what it reads or other outputs, but d2c_pg_rotate may work in place: refused
 *     with D2C_EINVAL, each buffer counted from its first element to its last;
 *   - T is float (D2C_F32) or bfloat16 (D2C_BF16), as the handle's dtype says: caches, queries and outputs;
 *   - pointers to rows and pages are multiples of 16 bytes, and so are row pitches (`_ld`, in elements); others of their
 *     element's size (D2C_EINVAL).
 *
 * The cache of a layer is n_pages pages of page_rows rows, K and V apart; page p, kv head h starts at element
 * (p * n_kv_heads + h) * page_rows * D (D = head_dim, E = 16 bytes of T: 8 for bfloat16, 4 for float).  From there, rows
 * 32u .. 32u + 31 lie in 32 * D elements, row 32u + t and dimension d
 *   K at (d / E) * 32 * E + slot(t) * E + d % E      slot(t) = t for float, t with its bits 2 and 3 exchanged for bfloat16
 *   V at (t / E) * D * E + d * E + t % E
 * Pages need no initial values: what was not appended is not looked at.
 *
 * A batch is n_rows packed rows: sequence b has rows row_start[b] .. row_start[b + 1] - 1 (none is legal), and its cache
 * rows 0 .. length[b] - 1 lie in pages pages[b, 0], pages[b, 1], ...  Row r of a sequence of m rows stands for index
 * at[r], or where at is NULL for the sequence's last rows: length - m + (r - row_start[b]).  Sequences may share pages.
 * On the device, where no error can be returned:
 *   - a length counts as at least 0 and at most page_cols * page_rows;
 *   - a page number outside [0, n_pages) is a page that is not there: its rows are not written, and not seen;
 *   - a negative origin counts as 0;
 *   - rows before row_start[0] and from row_start[batch] on belong to no sequence and are left as they are; row starts
 *     outside [0, n_rows] or not ascending leave all outputs and the caches undefined, and nothing else.
 * What d2c_pg_attention launches goes by the host's numbers, page_cols * page_rows among them, as lengths are known on the device only: where
 * sequences are short beside their table, a narrower one can save a launch or two (a call takes its own page_cols; rows of pages [batch, page_cols]).
 */
#ifndef D2C_PG_H
#define D2C_PG_H

#include <stdint.h>

#include "d2c.h"

#ifdef __cplusplus
extern "C" {
#endif

#define D2C_PG_MAX_PAIRS 64
#define D2C_PG_HALVES 0       /* pair i of a head is its dimensions (i, n_pairs + i) */
#define D2C_PG_NEIGHBOURS 1   /* (2 i, 2 i + 1)                                      */

typedef struct d2c_pg d2c_pg;   /* opaque; created by d2c_pg_init, freed by d2c_pg_destroy */

typedef struct {
  int32_t n_heads, n_kv_heads, head_dim;   /* head_dim 64 or 128; n_heads a multiple of n_kv_heads, up to 1024      */
  int32_t dtype;       /* D2C_F32 or D2C_BF16                                                                      */
  int32_t page_rows;   /* 32, 64, 128 or 256                                                                       */
  int32_t max_rows;    /* n_rows of one d2c_pg_attention call, up to 2^20; 0 = it is not used                      */
  int32_t max_batch;   /* sequences of one call, up to 1024; 0 = 1                                                 */
  int32_t n_pairs;     /* rotated pairs of a head: a multiple of 8 up to head_dim / 2 (further dimensions stay as
                          they are); 0 = no rotation                                                               */
  int32_t n_axes;      /* axes of a position, 1 to 4; 0 = 1                                                        */
  int32_t pairing;     /* D2C_PG_HALVES or D2C_PG_NEIGHBOURS                                                       */
  double  freq[D2C_PG_MAX_PAIRS];   /* pair i turns by freq[i] * position[axis[i]]; magnitudes up to 2^16          */
  uint8_t axis[D2C_PG_MAX_PAIRS];   /* below n_axes                                                                */
} d2c_pg_dims;

/* Pages of one layer's cache, caller-owned. */
typedef struct {
  void* k;             /* T, n_pages pages */
  void* v;
  int32_t n_pages;     /* at least 1 */
} d2c_pg_cache;

typedef struct {
  const int32_t* row_start;   /* [batch + 1] ascending                                           */
  const int32_t* length;      /* [batch] rows of the cache, those that the call appends included */
  const int32_t* pages;       /* [batch, page_cols]                                              */
  const int32_t* at;          /* [n_rows] index of each row in its sequence, or NULL (as above)  */
  const int32_t* origin;      /* [batch] where a sequence's mask blocks start, or NULL (0)       */
  int32_t batch, n_rows;      /* (host) n_rows up to 2^24                                        */
  int32_t page_cols;          /* (host) page_cols * page_rows up to 2^30                         */
} d2c_pg_batch;

int d2c_pg_init(const d2c_pg_dims* dims, d2c_pg** out);
int d2c_pg_destroy(d2c_pg* ctx);
/* Text of the last error of this handle (ctx NULL: of this thread's last d2c_pg_init that failed). */
const char* d2c_pg_last_error(const d2c_pg* ctx);
/* Bytes of device workspace the handle holds. */
int64_t d2c_pg_workspace_bytes(const d2c_pg* ctx);
/* Bytes of n_pages pages of K (V: as many). */
int d2c_pg_cache_size(const d2c_pg* ctx, int64_t n_pages, int64_t* bytes);

/* Rows turned by their positions: x (x_dtype: D2C_F32 or the handle's) [n, heads * D] with x_ld elements from row to row ->
 * out T, likewise.  pos [n_axes, n]: any int32.  The pair (a, b) of dimensions becomes (a cos w - b sin w, b cos w + a sin w),
 * w = freq * position; angles are formed in 64 bits, the rotation in fp32, rounded once.  inverse != 0 turns by -w: undoes
 * it, and is the gradient of x for one of out.  x may be out (same type and pitch).  n up to 2^24. */
int d2c_pg_rotate(d2c_pg* ctx, const void* x, int64_t x_ld, int32_t x_dtype, int32_t n, int32_t heads, const int32_t* pos,
                  int32_t inverse, void* out, int64_t out_ld, void* stream);

/* Rows k, v [n_rows, n_kv_heads * D] (dtype: D2C_F32 or the handle's) go into the pages of their sequences, k turned by the
 * rows' positions, rounded once; q [n_rows, n_heads * D], if given, is turned likewise into q_out T.  pos [n_axes, n_rows], or
 * NULL: each row's index, on every axis.  Without a rotation (n_pairs = 0) rows go as they are.  Rows whose index is outside
 * [0, length) go into no page.  Two rows of a call for one place of the cache leave its contents undefined. */
typedef struct {
  const void *q, *k, *v;          /* q may be NULL */
  int64_t q_ld, k_ld, v_ld;
  int32_t dtype;                  /* of q, k and v */
  const int32_t* pos;
  void* q_out;
  int64_t q_out_ld;
} d2c_pg_new;
int d2c_pg_append(d2c_pg* ctx, const d2c_pg_cache* cache, const d2c_pg_batch* batch, const d2c_pg_new* rows, void* stream);

/* Values of the cache rows that the batch's rows stand for: out_k / out_v T [n_rows, n_kv_heads * D] (either may be NULL).  An index outside
 * [0, length) or without a page gives zeros. */
int d2c_pg_read(d2c_pg* ctx, const d2c_pg_cache* cache, const d2c_pg_batch* batch, void* out_k, int64_t k_ld, void* out_v,
                int64_t v_ld, void* stream);

/* Attention of each row of q T [n_rows, n_heads * D] against its sequence's cache rows: out T, likewise.  Head h reads kv head
 * h / (n_heads / n_kv_heads).  The row of index i sees the rows j in [0, length) that are there, and of them
 *   block = 0   all;   block = B > 0   those below the end of i's block: blocks of B rows are counted from origin, the rows
 *               before it are one block (B = 1: causal;  B = block length: blocks that see each other in whole);
 *   window = W > 0   only j > i - W, and without blocks only j < i + W.
 * A row with a negative index sees nothing, unless neither at, block nor window is given.  A row that sees nothing gets zeros.
 * What a row does not see (NaN and infinities among it) does not change its result.
 * Scores are q k^T * scale (0: 1 / sqrt(D)); scores, softmax and sums are fp32; scores are meant to stay below 2^100 in magnitude.
 * bfloat16: probabilities are rounded to bfloat16 for the product with V, their sum is not.
 * The same call gives the same bits; with other sequences beside it, a sequence's sums can be split otherwise.
 * attn_avg float [n_rows, avg_ld], or NULL: columns below the sequence's length (and avg_ld) get the mean over the heads of the
 * softmax rows, 0 where the row sees nothing; columns behind are left as they are. */
typedef struct {
  const void* q;
  int64_t q_ld;
  void* out;
  int64_t out_ld;
  float* attn_avg;
  int64_t avg_ld;                 /* at most 2^30 */
  int32_t block, window;          /* 0 = none; up to 2^30 */
  float scale;                    /* positive, at most 2^127; 0 = 1 / sqrt(D) */
} d2c_pg_attend;
int d2c_pg_attention(d2c_pg* ctx, const d2c_pg_cache* cache, const d2c_pg_batch* batch, const d2c_pg_attend* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* D2C_PG_H */
