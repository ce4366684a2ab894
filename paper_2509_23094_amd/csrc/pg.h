// Launch interface of the paged cache's kernels (see include/d2c_pg.h), and what their device code shares.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "pg_plan.h"

namespace d2c {

constexpr int kPgUnit = 32;              // cache rows of one matrix-core tile: pages hold whole units
constexpr int kPgMaxBatch = 1024;
constexpr int kPgMaxSplits = 64;

struct PgShape { int H, Hkv, D, dtype, page_log2; };
struct PgRotation {                      // a kernel argument
  double turns[64];                      // revolutions per unit of position: freq / (2 pi)
  uint8_t axis[64];
  int n_pairs, n_axes, pairing;
};
struct PgBatch {
  const int32_t *row_start, *length, *pages, *at, *origin;
  int batch, n_rows, page_cols;
};
struct PgPages { void *k, *v; int n_pages; };

struct PgRows {                          // rows in, and where they go
  const void *q, *k, *v;
  int64_t q_ld, k_ld, v_ld, q_out_ld;
  const int32_t* pos;
  void* q_out;
  int src_dtype, q_heads;
  float sign;                            // -1 turns back
};
// batch null: q alone, by pos
hipError_t launch_pg_rows(const PgShape& s, const PgRotation& rot, const PgPages& pages, const PgBatch* batch, int n, const PgRows& rows,
                          hipStream_t st);
hipError_t launch_pg_read(const PgShape& s, const PgPages& pages, const PgBatch& batch, void* out_k, int64_t k_ld, void* out_v, int64_t v_ld,
                          hipStream_t st);

struct PgAttend {
  const void* q;
  void* out;
  float* avg;
  int64_t q_ld, out_ld, avg_ld;
  int block, window;
  float scale;
};
struct PgWorkspace {                     // sizes in pg_workspace
  int parts;                             // partial tiles of 32 rows
  size_t part_o, part_ml, row_ml, info, bytes;
};
PgWorkspace pg_workspace(const PgShape& s, int max_rows, int max_batch);
hipError_t launch_pg_attention(const PgShape& s, const PgPages& pages, const PgBatch& batch, const PgAttend& a, const PgWorkspace& w, void* ws,
                               int cus, hipStream_t st);

#ifdef __HIPCC__
// Row t of a unit -> its place among K's 16-byte pieces, so that the accumulators of S^T = K Q^T hold the keys in the order in which V lies
template <typename T> __device__ __forceinline__ int pg_slot(int t) { return t; }
template <> __device__ __forceinline__ int pg_slot<bf16>(int t) { return (t & 19) | (t & 4) << 1 | (t & 8) >> 1; }

// The sequence of packed row r and what it says of the row; the whole wave asks for one row.  Starts and lengths arrive in one round of loads.
struct PgRowAt {
  int seq, index, length;                // seq -1: the row belongs to none
  int first, count;                      // rows of the sequence
};
__device__ __forceinline__ PgRowAt pg_row_at(const PgBatch& b, int r, int page_log2) {
  const int lane = threadIdx.x & 63;
  int seq = 0, first = 0, next = 0, len = 0;
  for (int s0 = 0; s0 < b.batch; s0 += 64) {
    const int s = min(s0 + lane, b.batch - 1);
    const int lo = b.row_start[s], hi = b.row_start[s + 1], n = b.length[s];
    const uint64_t behind = __ballot(s0 + lane < b.batch && hi <= r);
    seq += __popcll(behind);
    const int mine = seq - s0;           // the first that ends behind r, if it is one of these
    if (mine < 64) {
      first = __shfl(lo, mine, 64);
      next = __shfl(hi, mine, 64);
      len = __shfl(n, mine, 64);
      break;
    }
  }
  PgRowAt a{-1, 0, 0, 0, 0};
  if (seq >= b.batch || r < first || r >= next || first < 0 || next > b.n_rows) return a;
  a.seq = seq;
  a.first = first;
  a.count = next - first;
  a.length = max(0, min(len, b.page_cols << page_log2));
  a.index = b.at ? b.at[r] : a.length - (next - first) + (r - first);
  return a;
}
#endif

}  // namespace d2c
