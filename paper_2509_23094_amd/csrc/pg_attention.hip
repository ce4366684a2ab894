// Attention of the packed rows of a batch over their sequences' pages (see include/d2c_pg.h).
//
// For each kv head the m rows of a sequence and the G = H / Hkv heads that share it make R = m G queries, taken 32 at a time.  A wave forms
// S^T[32 keys x 32 queries] = K Q^T and O^T[D x 32 queries] += V^T P^T with 32 x 32 matrix instructions.  An accumulator of S^T holds, for one query,
// the keys in just the order in which V lies in its pages, so the probabilities never leave registers; and both K's and V's operands lie
// there as 16 bytes a lane, so a unit of 32 rows is loaded in whole lines, whatever page it is in.
//   softmax in base 2 with a reference per query that is raised only when a score passes it by 2^8 (the result is the same softmax); sums in
//   fp32 before probabilities are rounded to T for the second product.
//   masks: query r sees the keys lo_r <= j < hi_r.  Keys outside some query's range are looked at again (scores set to -inf, V zeroed where no
//   query sees it); elsewhere there is no mask.  What is not finite in such a unit's V (0 times it would be NaN) is left out of the product and
//   added by itself where a query sees it.
// The keys of a tile are split over workgroups where tiles alone would not fill the chip; each split leaves its reference, sum and
// unnormalised O, and a second launch joins them in order.  Which workgroup does what is computed on the device from the row starts and lengths, by every
// workgroup for itself (plan), so that a captured call follows them.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "internal.h"
#include "pg.h"

namespace d2c {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kFloor = -3.0e38f;      // a reference that no score has raised: finite, so that differences with it are no NaN
constexpr float kRaise = 8.f;

// n / d for n below 2^30 without a division (one takes a wave a quarter of a microsecond): m = ceil(2^(32 + s) / d) is less than d / 2^(32 + s) above
// the quotient, which n d < 2^(32 + s) 2^30 / 2^31 does not notice; powers of two (m = 0) are shifts.
struct Div { uint32_t m; int s; };
inline Div div_by(uint32_t d) {
  int s = 0;
  while ((uint64_t)2 << s <= d) ++s;
  return Div{(d & (d - 1)) == 0 ? 0u : (uint32_t)((((uint64_t)1 << (32 + s)) + d - 1) / d), s};
}
__device__ __forceinline__ int operator/(int n, const Div& d) { return (int)((d.m ? __umulhi((uint32_t)n, d.m) : (uint32_t)n) >> d.s); }

struct AttendArgs {
  PgBatch batch;
  PgPages pages;
  const void* q;
  void* out;
  int64_t q_ld, out_ld;
  int H, Hkv, G, page_log2, block, window;
  Div by_hkv, by_g;
  float c2;                      // scale * log2(e)
  float much, together;          // work (see work_of) from which on a sequence is for the kernel for many queries: its own, that of all that fill tiles
  int max_splits, part_first, part_limit;      // partial tiles of this launch
  float* part_o;                 // [part][32][D]
  float2* part_ml;               // [part][32]: reference, sum
  float2* row_ml;                // [row][H]: reference, 1 / sum (where the average is wanted), or null
  int4* info;                    // [sequence]: splits | first part << 8, tiles of 32 queries that are split, first row, rows
};

// All cache lines of the arguments at once: as they are needed one by one, each first use of a line waits for memory.
__device__ __forceinline__ void fetch_arguments(const AttendArgs& a) {
  asm volatile("" ::"s"(a.batch.row_start), "s"(a.batch.page_cols), "s"(a.pages.n_pages), "s"(a.out_ld), "s"(a.H), "s"(a.window), "s"(a.by_g.s), "s"(a.c2),
               "s"(a.part_limit), "s"(a.part_ml), "s"(a.info));
}

// ------------------------------------------------------------------ the plan

struct PlanSeq { int row0, m, length, unit0; };     // unit0: first unit that a row of the sequence can see
struct Plan {
  PlanSeq* seq;                  // [batch]
  int* first;                    // [batch + 1] first item
  int* split;                    // [batch] splits << 24 | first partial tile
  int* whole;                    // [batch] tiles that are not split: the last ones, which come first
  int chunk, items;              // units of a split
  // of a few sequences: lane b's own of the above, so that an item is found without LDS
  bool solo;
  PlanSeq my;
  int my_first, my_end, my_split, my_whole;
};
inline size_t plan_bytes(int batch) { return (size_t)batch * (sizeof(PlanSeq) + 12) + 16; }

// Reductions and scans over the wave by data-parallel moves within it (a shuffle through LDS takes ten times as long, and a plan is all
// latency).  Inclusive scan: lane 63 ends with the whole.
template <int CTRL, int ROWS> __device__ __forceinline__ int moved(int v, int none) { return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xf, false); }
template <typename F> __device__ __forceinline__ int scan(int v, int none, F f) {
  v = f(v, moved<0x111, 0xf>(v, none));        // row_shr 1, 2, 4, 8: within 16 lanes
  v = f(v, moved<0x112, 0xf>(v, none));
  v = f(v, moved<0x114, 0xf>(v, none));
  v = f(v, moved<0x118, 0xf>(v, none));
  v = f(v, moved<0x142, 0xa>(v, none));        // lane 15 of a row to the next row, lane 31 to the upper half
  v = f(v, moved<0x143, 0xc>(v, none));
  return v;
}
__device__ __forceinline__ int scan_sum(int v) { return scan(v, 0, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ int reduce_max(int v) { return last_lane(scan(v, INT32_MIN, [](int a, int b) { return max(a, b); })); }
__device__ __forceinline__ int reduce_min(int v) { return last_lane(scan(v, INT32_MAX, [](int a, int b) { return min(a, b); })); }

// An item is (tile of TILES * 32 queries, split, kv head) of a sequence; kv heads run fastest, so that tiles that read the same keys are a
// multiple of Hkv workgroups apart (on one XCD where that is a multiple of 8).  As many tiles as fill whole rounds of workgroups are not split (a
// sequence's last ones, which a mask leaves the most keys, come first); the rest is, in splits of equal length for all sequences: of 1 .. 64 for the
// longest sequence, each lane of a wave takes one and estimates the time as rounds of workgroups times (units of a split + what an item costs besides:
// as much as 32 units of the kernel for few, 8 of the one for many; with 8 for few, 200 tokens on 1500 keys each took 92 us, with 32 they take 81), and what the partial
// results cost, 128 KB out and in for an item of the kernel for many (0.06 units: 1024 rows of 28 heads on 16000 keys 318 -> 247 us, 1500 of 32 on 8000 235 -> 216).
template <int TILES> __device__ __forceinline__ int tiles_in(int queries) { return (queries + 32 * TILES - 1) / (32 * TILES); }
// About how many (query, key) pairs a sequence has
__device__ __forceinline__ float work_of(const AttendArgs& a, int m, int length) {
  float keys = (float)length;
  if (a.block > 0 && !a.batch.at) keys = fmaxf(keys - 0.5f * (float)m, 0.5f * keys);
  if (a.window > 0) keys = fminf(keys, (float)a.window * (a.block > 0 ? 1.f : 2.f));
  return (float)m * (float)a.H * keys;
}
// tiles of 32 queries of a sequence that are split: the first ones
template <int TILES> __device__ __forceinline__ int split_tiles(int queries, int whole) {
  return min((queries + 31) / 32, (tiles_in<TILES>(queries) - whole) * TILES);
}
// A sequence goes to the kernel for many queries by its own work; or together with at least three others that fill their tiles there, by the work of all of
// them (a sum of whole numbers, counted above it: both kernels have to come to the same).
constexpr float kWorkUnit = 65536.f;
constexpr int kOne = 1 << 21;
__device__ __forceinline__ int share_of_work(const AttendArgs& a, int m, int length) {
  const int R = m * a.G, tiles = (R + 255) / 256;
  const int n = (int64_t)10 * R >= (int64_t)7 * 256 * tiles ? (int)fminf(work_of(a, m, length) / kWorkUnit, 1024.f) : 0;
  return n > 0 ? n + kOne : 0;
}
__device__ __forceinline__ bool has_much(const AttendArgs& a, int m, int length, bool together) {
  return work_of(a, m, length) > a.much || (together && (float)(share_of_work(a, m, length) % kOne) * kWorkUnit > a.together / 64.f);
}
template <int TILES, int THREADS>
__device__ __forceinline__ Plan make_plan(const AttendArgs& a, unsigned char* lds, float item_cost, float part_cost) {
  constexpr int kWaves = THREADS / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, batch = a.batch.batch, G = a.G;
  Plan p;
  p.seq = reinterpret_cast<PlanSeq*>(lds);
  p.first = reinterpret_cast<int*>(lds + (size_t)batch * sizeof(PlanSeq));
  p.split = p.first + batch + 1;
  p.whole = p.split + batch;
  __shared__ float load[kWaves][64];
  __shared__ int most[kWaves], rows_of[kWaves], tiles_of[kWaves];
  // a few sequences: each wave does it all by itself (they write the same values), without a barrier
  const bool solo = batch <= 16;
  p.solo = solo;
  p.my = PlanSeq{0, 0, 0, 0};
  bool together = false;
  if (a.together < 3e38f) {
    uint32_t sum = 0;                  // (1024 sequences: 2^31)
    for (int b = solo ? lane : tid; b < batch; b += THREADS) {
      const int m = pg_span(a.batch.row_start[b], a.batch.row_start[b + 1], a.batch.n_rows).m;
      sum += (uint32_t)share_of_work(a, m, max(0, min(a.batch.length[b], a.batch.page_cols << a.page_log2)));
    }
    sum = (uint32_t)last_lane(scan_sum((int)sum));
    if (!solo) {
      if (lane == 0) most[wave] = (int)sum;
      __syncthreads();
      sum = 0;
      for (int w = 0; w < kWaves; ++w) sum += (uint32_t)most[w];
      __syncthreads();
    }
    together = sum / kOne >= 4 && (float)(sum % kOne) * kWorkUnit > a.together;
  }
  int units = 0, rows = 0, tiles = 0;
  for (int b = solo ? lane : tid; b < batch; b += THREADS) {
    const int lo = a.batch.row_start[b], hi = a.batch.row_start[b + 1], len = a.batch.length[b];
    PlanSeq s;
    const PgSpan span = pg_span(lo, hi, a.batch.n_rows);
    s.row0 = span.row0;
    s.m = span.m;
    s.length = max(0, min(len, a.batch.page_cols << a.page_log2));
    rows = min(rows + s.m, 1 << 22);             // (starts that are not ascending: the sum tells; n_rows is 2^20 at most)
    if (has_much(a, s.m, s.length, together) != (TILES > 1)) s.m = 0;
    tiles = min(tiles + tiles_in<TILES>(s.m * G), 1 << 25);
    s.unit0 = a.window > 0 && !a.batch.at ? max(0, s.length - s.m - a.window + 1) / kPgUnit : 0;
    p.seq[b] = p.my = s;
    if (s.m > 0) units = max(units, (s.length + kPgUnit - 1) / kPgUnit - s.unit0);
  }
  units = max(1, reduce_max(units));
  rows = last_lane(scan_sum(rows));
  int all = last_lane(scan_sum(tiles));
  if (!solo) {
    if (lane == 0) { most[wave] = units; rows_of[wave] = rows; tiles_of[wave] = all; }
    __syncthreads();
    rows = all = 0;
    for (int w = 0; w < kWaves; ++w) {
      units = max(units, most[w]);
      rows = min(rows + rows_of[w], 1 << 22);
      all = min(all + tiles_of[w], 1 << 25);
    }
  }
  const bool sane = rows <= a.batch.n_rows;
  all *= a.Hkv;
  const float share = all < (int)gridDim.x ? 0.f : (float)(all / (int)gridDim.x * (int)gridDim.x) / (float)all + 1e-6f;      // of tiles that stay whole
  const int chunk = (units + lane) / (lane + 1);          // of lane + 1 splits
  const float inv = 1.f / (float)chunk;
  float items = 0.f;
  for (int b = solo ? 0 : wave; b < batch; b += solo ? 1 : kWaves) {
    const PlanSeq s = p.seq[b];
    const int tiles = tiles_in<TILES>(s.m * G), n = (s.length + kPgUnit - 1) / kPgUnit - s.unit0;
    items += (float)(tiles - pg_whole(tiles, share)) * fmaxf(1.f, ceilf((float)n * inv - 1e-3f));
  }
  float cost = items * (float)a.Hkv;
  if (!solo) {
    load[wave][lane] = cost;
    __syncthreads();
    cost = 0.f;
    for (int w = 0; w < kWaves; ++w) cost += load[w][lane];
  }
  cost = ceilf(cost / (float)gridDim.x) * ((float)chunk + item_cost) + (lane > 0 ? part_cost * cost : 0.f);
  // the cheapest, of equal ones the fewest splits (a positive float's bits are in its order)
  const int bits = lane < a.max_splits ? __builtin_bit_cast(int, cost) : INT32_MAX;
  const int best = reduce_min(bits);
  p.chunk = __builtin_amdgcn_readlane(chunk, (int)__builtin_ctzll(__ballot(bits == best)));
  if (solo || wave == 0) {
    int item = 0, part = a.part_first;
    for (int b0 = 0; b0 < batch; b0 += 64) {
      const int b = b0 + lane;
      int n_tiles = 0, n_parts = 0, splits = 1, n_whole = 0;
      if (b < batch && sane) {
        const PlanSeq s = p.seq[b];
        n_tiles = tiles_in<TILES>(s.m * G);
        n_whole = pg_whole(n_tiles, share);
        const int n = (s.length + kPgUnit - 1) / kPgUnit - s.unit0;
        splits = max(1, (n + p.chunk - 1) / p.chunk);
        const int64_t parts = (int64_t)min((s.m * G + 31) / 32, (n_tiles - n_whole) * TILES) * a.Hkv * splits;
        n_parts = splits > 1 ? (int)min(parts, (int64_t)1 << 24) : 0;
      }
      const int at_part = scan_sum(n_parts);
      // a sequence whose parts have no room is not split
      const bool fits = part + at_part <= a.part_limit;
      if (!fits) splits = 1;
      if (splits == 1) n_whole = n_tiles;
      const int n_items = (n_whole + (n_tiles - n_whole) * splits) * a.Hkv;
      const int at_item = scan_sum(n_items);
      p.my_end = item + at_item;
      p.my_first = p.my_end - n_items;
      p.my_whole = n_whole;
      p.my_split = splits << 24 | (splits > 1 ? part + at_part - n_parts : 0);
      if (b < batch) {
        p.first[b] = p.my_first;
        p.whole[b] = n_whole;
        p.split[b] = p.my_split;
      }
      item += last_lane(at_item);
      part = min(part + last_lane(at_part), 1 << 28);
    }
    if (lane == 0) p.first[batch] = item;
  }
  if (solo) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  else __syncthreads();
  p.items = solo ? last_lane(p.my_end) : p.first[batch];
  // what the join reads, of every sequence anew: by the launch that has its rows, of one without rows (none within the batch's: p.seq alone
  // does not tell) by each launch, with no tiles.  A record that stays would be an earlier call's, with rows that this one may not have.
  if (blockIdx.x == 0)
    for (int b = tid; b < batch; b += THREADS)
      if (p.seq[b].m > 0 || pg_span(a.batch.row_start[b], a.batch.row_start[b + 1], a.batch.n_rows).m == 0)
        a.info[b] = make_int4(p.split[b] >> 24 | (p.split[b] & 0xffffff) << 8, split_tiles<TILES>(p.seq[b].m * G, p.whole[b]), p.seq[b].row0, p.seq[b].m);
  return p;
}
// Of the sequence that an item belongs to (as many as end at or before it): all that the item's work needs
struct Found { int b, first, split, whole; PlanSeq seq; };
__device__ __forceinline__ Found find(const Plan& p, int batch, int item) {
  const int lane = threadIdx.x & 63;
  Found f;
  if (p.solo) {
    f.b = __popcll(__ballot(lane < batch && p.my_end <= item));
    auto of = [&](int mine) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(mine, f.b); };
    f.first = of(p.my_first);
    f.split = of(p.my_split);
    f.whole = of(p.my_whole);
    f.seq = PlanSeq{of(p.my.row0), of(p.my.m), of(p.my.length), of(p.my.unit0)};
    return f;
  }
  f.b = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) f.b += __popcll(__ballot(b0 + lane < batch && p.first[b0 + min(lane, batch - 1 - b0) + 1] <= item));
  f.first = p.first[f.b];
  f.split = p.split[f.b];
  f.whole = p.whole[f.b];
  f.seq = p.seq[f.b];
  return f;
}

// Where an item of a sequence is: tile, split, kv head
struct Place { int tile, hk, split, splits; };
template <int TILES> __device__ __forceinline__ Place place_of(const AttendArgs& a, const Found& f, int item) {
  const int local = item - f.first, whole = f.whole, tiles = tiles_in<TILES>(f.seq.m * a.G), splits = f.split >> 24;
  const int at = local / a.by_hkv;
  Place w;
  w.hk = local - at * a.Hkv;
  w.splits = 1;
  w.split = 0;
  w.tile = tiles - 1 - at;
  if (at >= whole) {                     // below 2^14 (there are no more partial tiles): the quotient in fp32 is off by one at the most
    const int n = at - whole;
    int t = (int)((float)n * __builtin_amdgcn_rcpf((float)splits));
    t -= n < t * splits;
    t += n >= (t + 1) * splits;
    w.splits = splits;
    w.split = n - t * splits;
    w.tile = tiles - 1 - whole - t;
  }
  w.hk = __builtin_amdgcn_readfirstlane(w.hk);
  w.splits = __builtin_amdgcn_readfirstlane(w.splits);
  w.split = __builtin_amdgcn_readfirstlane(w.split);
  w.tile = __builtin_amdgcn_readfirstlane(w.tile);
  return w;
}

// Keys that a row of index i sees: lo <= j < hi, lo > hi - 1 where there are none
__device__ __forceinline__ void visible(const AttendArgs& a, int i, int origin, int length, int& lo, int& hi) {
  lo = 0;
  hi = length;
  if (a.block > 0) {
    const int64_t end = i < origin ? origin : origin + ((int64_t)(i - origin) / a.block + 1) * a.block;
    hi = (int)min((int64_t)length, end);
  }
  if (a.window > 0) {
    lo = (int)max((int64_t)0, (int64_t)i - a.window + 1);
    if (a.block == 0) hi = (int)min((int64_t)length, (int64_t)i + a.window);
  }
  if (i < 0 && (a.batch.at || a.block > 0 || a.window > 0)) hi = 0;
  if (lo >= hi) { lo = 0x7fffffff; hi = 0; }
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// acc += A B^T over a pair of 16-byte pieces per lane: 16 (float: 8) along the contraction
template <typename T> __device__ __forceinline__ f32x16 mm(const u32x4& a, const u32x4& b, f32x16 acc);
template <> __device__ __forceinline__ f32x16 mm<bf16>(const u32x4& a, const u32x4& b, f32x16 acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mm<float>(const u32x4& a, const u32x4& b, f32x16 acc) {
  const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], acc, 0, 0, 0);
  return acc;
}
// key of accumulator element i, within a unit
template <typename T> __device__ __forceinline__ int key_of(int i, int g) { return sizeof(T) == 2 ? 16 * (i >> 3) + 8 * g + (i & 7) : 8 * (i >> 2) + 4 * g + (i & 3); }
// Probabilities as operands: pieces s = 0 .. 16 / E - 1.  bf16: rounded to it (half a step, 2^-8 of each), because the matrix instruction takes both operands in one type
// and the other is V; their sum, the references and O stay in fp32.  Outputs of the timed cases are off by 1.6 - 2.0e-3 (norm) against 64 bits, where fp32
// probabilities and the output's own rounding leave 1.6 - 1.7e-3; a second piece for what the rounding leaves would be half as many products again.
template <typename T> __device__ __forceinline__ u32x4 p_piece(const float (&x)[16], int s);
template <> __device__ __forceinline__ u32x4 p_piece<bf16>(const float (&x)[16], int s) {
  return u32x4{pack2(x[8 * s], x[8 * s + 1]), pack2(x[8 * s + 2], x[8 * s + 3]), pack2(x[8 * s + 4], x[8 * s + 5]), pack2(x[8 * s + 6], x[8 * s + 7])};
}
template <> __device__ __forceinline__ u32x4 p_piece<float>(const float (&x)[16], int s) {
  return __builtin_bit_cast(u32x4, f32x4{x[4 * s], x[4 * s + 1], x[4 * s + 2], x[4 * s + 3]});
}
// a piece of V with the elements of keys outside [lo, hi) zeroed; key: of its first element
template <typename T> __device__ __forceinline__ u32x4 keep_keys(u32x4 v, int key, int lo, int hi) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int k = key + 2 * w;
      v[w] &= (k >= lo && k < hi ? 0xffffu : 0u) | (k + 1 >= lo && k + 1 < hi ? 0xffff0000u : 0u);
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] = key + w >= lo && key + w < hi ? v[w] : 0u;
  }
  return v;
}
// zeroes what is not finite; true if there was something
template <typename T> __device__ __forceinline__ bool drop_not_finite(u32x4& v) {
  bool any = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 2) {
      const bool lo = (v[w] & 0x7f80u) == 0x7f80u, hi = (v[w] & 0x7f800000u) == 0x7f800000u;
      any = any || lo || hi;
      v[w] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    } else {
      const bool bad = (v[w] & 0x7f800000u) == 0x7f800000u;
      any = any || bad;
      v[w] = bad ? 0u : v[w];
    }
  }
  return any;
}

// The 32 queries of a tile, one per lane and half: where they are, what they see
struct Queries {
  int row, head, lo, hi;          // lo, hi: this lane's query
  bool valid;
  int all_lo, all_hi;             // what any of them sees lies within
  int both_lo, both_hi;           // what all of them see
};
__device__ __forceinline__ Queries queries_of(const AttendArgs& a, const PlanSeq& s, int b, int hk, int first, int r32) {
  const int G = a.G, R = s.m * G;
  Queries q;
  const int r = first + r32;
  q.valid = r < R;                        // past the last: the tile's first query again, not stored
  const int use = q.valid ? r : first;
  q.row = use / a.by_g;
  q.head = hk * G + (use - q.row * G);
  q.row += s.row0;
  const int i = a.batch.at ? a.batch.at[q.row] : s.length - s.m + (q.row - s.row0);
  visible(a, i, a.batch.origin ? max(0, a.batch.origin[b]) : 0, s.length, q.lo, q.hi);
  q.all_lo = reduce_min(q.lo);
  q.both_lo = reduce_max(q.lo);
  q.all_hi = reduce_max(q.hi);
  q.both_hi = reduce_min(q.hi);
  return q;
}

// A unit's scores, -inf where the query does not see the key
template <typename T> __device__ __forceinline__ void mask_unit(f32x16& x, bool edge, int key0, const Queries& q) {
  const int g = (threadIdx.x & 63) >> 5;
  if (edge) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = key0 + key_of<T>(i, g);
      x[i] = key >= q.lo && key < q.hi ? x[i] : -INFINITY;
    }
  }
}
__device__ __forceinline__ float top_of(const f32x16& x) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  return top;
}
// o and l are relative to 2^ref, which is raised only where a score (top: this lane's largest) passes it by more than kRaise
template <int DT> __device__ __forceinline__ void raise(float top, float c2, float& ref, float& l, f32x16 (&o)[DT]) {
  if (__ballot(top * c2 > ref + kRaise) == 0) return;
  top = fmaxf(top, __shfl_xor(top, 32, kWave)) * c2;
  const float to = top > ref + kRaise ? top : ref, alpha = exp2_hw(ref - to);
  ref = to;
  l *= alpha;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
}
// masked scores -> probabilities against the reference, as operands; their sum goes to l
template <typename T> __device__ __forceinline__ void exps_unit(const f32x16& s, float c2, float ref, float& l, u32x4 (&p)[kPgUnit / (32 / (int)sizeof(T))]) {
  float x[16], sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = exp2_hw(fmaf(s[i], c2, -ref));
    sum += x[i];
  }
  l += sum;
#pragma unroll
  for (int i = 0; i < kPgUnit / (32 / (int)sizeof(T)); ++i) p[i] = p_piece<T>(x, i);
}

// What is not finite in the rows of V that some of the queries see, for those that do: 0 times it would be NaN for the others, so products leave it out
// (V zeroed).  unit: V in memory.
template <typename T, int DT> __device__ __forceinline__ void add_not_finite(const T* unit, int key0, const Queries& q, f32x16 (&o)[DT]) {
  constexpr int E = 16 / sizeof(T);
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll 1
  for (int j = 0; j < kPgUnit; ++j) {
    const int key = key0 + j;
    if (key < q.all_lo || key >= q.all_hi) continue;
    const bool sees = key >= q.lo && key < q.hi;
    const T* row = unit + (j / E) * (32 * DT * E) + 4 * g * E + j % E;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = to_f32(row[(32 * dt + 8 * (i >> 2) + (i & 3)) * E]);
        o[dt][i] += sees && !(fabsf(y) <= 3.402823466e38f) ? y : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);       // a tile at a time: this rare path must not cost registers
    }
  }
}

// O^T += V^T P^T of one unit whose V pieces are in registers.  In an edge unit V is zeroed where no query sees it, and where it is not finite.
template <typename T, int DT>
__device__ __forceinline__ void values_unit(u32x4 (&v)[kPgUnit / (32 / (int)sizeof(T))][DT], const u32x4 (&p)[kPgUnit / (32 / (int)sizeof(T))], bool edge, int key0,
                                            const Queries& q, const T* unit, f32x16 (&o)[DT]) {
  constexpr int E = 16 / sizeof(T), NS = kPgUnit / (2 * E);
  const int g = (threadIdx.x & 63) >> 5;
  bool dropped = false;
  if (edge) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        v[s][dt] = keep_keys<T>(v[s][dt], key0 + (2 * s + g) * E, q.all_lo, q.all_hi);
        dropped = drop_not_finite<T>(v[s][dt]) || dropped;
      }
    dropped = __ballot(dropped) != 0;
  }
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = mm<T>(v[s][dt], p[s], o[dt]);
  if (__builtin_expect(dropped, 0)) add_not_finite<T, DT>(unit, key0, q, o);
}

template <typename T> __device__ __forceinline__ void store4(T* p, const f32x4& v);
template <> __device__ __forceinline__ void store4<bf16>(bf16* p, const f32x4& v) { *reinterpret_cast<u32x2*>(p) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])}; }
template <> __device__ __forceinline__ void store4<float>(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
// of a sum of exponentials: 0 where a row saw nothing, NaN stays
__device__ __forceinline__ float inverse_of(float sum) { return sum > 0.f ? 1.f / sum : sum; }

// ------------------------------------------------------------------ few queries: operands straight from the pages

// (query, key) pairs, all heads, from which on a sequence goes to the kernel for many queries.  us by the one for few and by it: bf16, 32 heads of 128, 8000
// keys: 256 rows (66e6) 66 and 58, 128 rows 43 and 47; 28 on 4, 4000 keys: 1024 rows (115e6) 105 and 90, 512 rows 57 and 59; 12 heads of 64 on 2, 16000 keys: 1024
// rows (197e6) 104 and 88, 512 rows 61 and 67; float, where both wait for the matrix cores, 32 heads, 2048 keys, 2000 rows, no mask 646 and 531, causal 376 and 533.
// Float has one threshold for what a mask does differently to the two: it keeps both of those calls in the kernel for few, which the causal one gains more by (157)
// than the other loses (115).
// Several sequences of bf16 heads of 128 together, from half of it on, but for those with less than a 64th of that (others: no gain).  Lengths falling evenly to a
// 20th, 28 heads on 4: 24 of 300 rows on 600 keys 104 and 87, 8 of 100 on 4000 82 and 66, 4 of 500 on 2000 83 and 71, but 12 of 400 on 1500, which nothing
// here tells apart from them, 124 and 134; 32 heads: 16 of 256 on 600 83 and 64, 6 of 700 on 2000 155 and 123; two of 512 on 2000, which stay where they are, 55
// and 69.  The host leaves the second launch out wherever rows times the page table's keys stay below the whole of it, so sequences that fill their tables and
// have between half of it and all of it together stay in the kernel for few.
template <typename T, int D> constexpr float kMuch = sizeof(T) == 4 ? 256e6f : D == 64 ? 128e6f : 64e6f;
constexpr int kManyWaves = 8, kFewWaves = 4;


// One tile of 32 queries per workgroup: its waves take the units of a split in turn and are merged through LDS.  K and V are used once, so nothing is staged:
// two workgroups a compute unit, each wave with the next unit's K or V on its way while it works on what has come.  Bound by memory where caches are long
// (64 tokens, 28 heads on 4, 279000 keys in all: 118 us, 4.8 TB/s, what a large copy reaches; one token, 60001 keys: 24 us, 5.0 TB/s, matrix cores 8 % and
// vector units 16 % busy), by its chain of dependent steps where they are short (1023 keys: 7 - 9 us, of which the plan 1.7).  The host takes eight waves instead
// of four where that saves the second launch.
template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void pg_few_kernel(const AttendArgs a) {
  constexpr int E = 16 / sizeof(T), DT = D / 32, NF = D / (2 * E), NS = kPgUnit / (2 * E);
  extern __shared__ __attribute__((aligned(16))) unsigned char plan_lds[];
  __shared__ f32x4 merge[kWaves][DT * 4][64];       // before: the queries
  u32x4 (*q_lds)[64] = reinterpret_cast<u32x4 (*)[64]>(&merge[0][0][0]);
  __shared__ float wref[kWaves][32], wl[kWaves][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, r32 = lane & 31;
  fetch_arguments(a);
  const Plan plan = make_plan<1, 64 * kWaves>(a, plan_lds, 32.f, 0.f);
  const int G = a.G;
  const size_t head_pitch = (size_t)D << a.page_log2;           // elements
  for (int item = blockIdx.x; item < plan.items; item += gridDim.x) {
    const Found found = find(plan, a.batch.batch, item);
    const int b = found.b;
    const PlanSeq s = found.seq;
    const Place at_item = place_of<1>(a, found, item);
    const int hk = at_item.hk, split = at_item.split, tile = at_item.tile, splits = at_item.splits;
    const Queries q = queries_of(a, s, b, hk, tile * 32, r32);
    // units of this split that a query sees; none: [0, 0)
    int u0 = s.unit0 + split * plan.chunk, u1 = splits == 1 ? 0x7fffffff : u0 + plan.chunk;
    if (splits == 1) u0 = 0;
    if (q.all_hi > 0) {
      u0 = max(u0, q.all_lo / kPgUnit);
      u1 = min(u1, (q.all_hi + kPgUnit - 1) / kPgUnit);
    } else u1 = u0;
    const int n_units = max(0, u1 - u0), n_mine = (n_units - wave + kWaves - 1) / kWaves;

    // the queries as operands, a wave's share, to LDS once the first unit is requested too
    constexpr int kMyQ = (NF + kWaves - 1) / kWaves;
    u32x4 my_q[kMyQ];
    const T* qrow = (const T*)a.q + (int64_t)q.row * a.q_ld + q.head * D + g * E;
#pragma unroll
    for (int i = 0; i < kMyQ; ++i) my_q[i] = ld16(qrow + min(wave + i * kWaves, NF - 1) * 2 * E);

    const int32_t* pages = a.batch.pages + (int64_t)b * a.batch.page_cols;
    int ids = 0;                              // page numbers of this wave's next 64 units
    auto page_of = [&](int k) {
      if ((k & 63) == 0) {
        const int u = min(u0 + wave + (k + lane) * kWaves, u1 - 1);
        ids = pages[u >> (a.page_log2 - 5)];
      }
      return __builtin_amdgcn_readlane(ids, k & 63);
    };
    u32x4 kr[NF], vr[NS][DT];
    auto unit_at = [&](int page, int u) __attribute__((always_inline)) {
      const int in = u & ((1 << (a.page_log2 - 5)) - 1);
      const int safe = (unsigned)page < (unsigned)a.pages.n_pages ? page : 0;
      return ((size_t)safe * a.Hkv + hk) * head_pitch + (size_t)in * kPgUnit * D;
    };
    const int k_lane = (g * kPgUnit + r32) * 16, v_lane = (g * D + r32) * 16;
    constexpr int kUnitBytes = kPgUnit * D * (int)sizeof(T);
    auto load_k = [&](size_t at) __attribute__((always_inline)) {
      const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((T*)a.pages.k + at, 0, kUnitBytes, 0x00020000);
#pragma unroll
      for (int f = 0; f < NF; ++f) kr[f] = __builtin_amdgcn_raw_buffer_load_b128(src, k_lane, f * (2 * kPgUnit * 16), 0);
    };
    auto load_v = [&](size_t at) __attribute__((always_inline)) {
      const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((T*)a.pages.v + at, 0, kUnitBytes, 0x00020000);
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[st][dt] = __builtin_amdgcn_raw_buffer_load_b128(src, v_lane, (2 * st * D + 32 * dt) * 16, 0);
    };
    // The next unit's K is requested as soon as this one's is used, V likewise.  Float heads of 128 have no registers for that: K when it is
    // needed, V behind the scores.
    constexpr bool kAhead = sizeof(T) == 2 || D == 64;
    int page = 0, next = 0;
    size_t at = 0, at_next = 0;
    if (n_mine > 0) {
      page = page_of(0);
      at = unit_at(page, u0 + wave);
      if (kAhead) {
        load_k(at);
        load_v(at);
      }
    }
#pragma unroll
    for (int i = 0; i < kMyQ; ++i)
      if (NF % kWaves == 0 || wave + i * kWaves < NF) q_lds[wave + i * kWaves][lane] = my_q[i];
    __syncthreads();

    f32x16 o[DT] = {};
    float ref = kFloor, l = 0.f;
    for (int k = 0; k < n_mine; ++k) {
      const int u = u0 + wave + k * kWaves, key0 = u * kPgUnit;
      const bool more = k + 1 < n_mine, there = (unsigned)page < (unsigned)a.pages.n_pages;
      if (more) {
        next = page_of(k + 1);
        at_next = unit_at(next, u + kWaves);
      }
      if (there) {
        const bool edge = key0 < q.both_lo || key0 + kPgUnit > q.both_hi;
        if (!kAhead) load_k(at);
        f32x16 acc = {};
#pragma unroll
        for (int f = 0; f < NF; ++f) acc = mm<T>(kr[f], q_lds[f][lane], acc);
        if (!kAhead) {
          __builtin_amdgcn_sched_barrier(0);
          load_v(at);
        } else if (more) load_k(at_next);
        u32x4 p[NS];
        mask_unit<T>(acc, edge, key0, q);
        raise<DT>(top_of(acc), a.c2, ref, l, o);
        exps_unit<T>(acc, a.c2, ref, l, p);
        values_unit<T, DT>(vr, p, edge, key0, q, (const T*)a.pages.v + at, o);
      } else if (kAhead && more) load_k(at_next);
      if (kAhead && more) load_v(at_next);
      page = next;
      at = at_next;
    }
    l += __shfl_xor(l, 32, kWave);

    // merge the waves that had a unit: each adds up some fours of neighbouring dimensions, 8 n + 4 g on with n = wave, wave + kWaves ..
    constexpr int kFours = DT * 4 / kWaves;
    const int n_waves = min(kWaves, n_units);
    __syncthreads();
    if (wave < n_waves) {
      if (g == 0) { wref[wave][r32] = ref; wl[wave][r32] = l; }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) merge[wave][dt * 4 + i][lane] = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    }
    __syncthreads();
    float top = kFloor, sum = 0.f, weight[kWaves];
    f32x4 y[kFours] = {}, part_of[kWaves][kFours];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      weight[w] = w < n_waves ? wref[w][r32] : kFloor;
#pragma unroll
      for (int n = 0; n < kFours; ++n) part_of[w][n] = w < n_waves ? merge[w][n * kWaves + wave][lane] : f32x4{};
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, weight[w]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      weight[w] = exp2_hw(weight[w] - top);
      sum += w < n_waves ? wl[w][r32] * weight[w] : 0.f;
#pragma unroll
      for (int n = 0; n < kFours; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) y[n][j] = fmaf(part_of[w][n][j], weight[w], y[n][j]);
    }
    const int d0 = 8 * wave + 4 * g;
    if (q.valid) {
      if (splits == 1) {
        const float inv = inverse_of(sum);
        T* to = (T*)a.out + (int64_t)q.row * a.out_ld + q.head * D + d0;
#pragma unroll
        for (int n = 0; n < kFours; ++n) store4<T>(to + 8 * kWaves * n, y[n] * inv);
        if (a.row_ml && wave == 0 && g == 0) a.row_ml[(size_t)q.row * a.H + q.head] = make_float2(top, inv);
      } else {
        const size_t part = (size_t)(found.split & 0xffffff) + ((size_t)hk * split_tiles<1>(s.m * G, found.whole) + tile) * splits + split;
        float* to = a.part_o + (part * 32 + r32) * D + d0;
        if (n_units > 0) {
#pragma unroll
          for (int n = 0; n < kFours; ++n) store4<float>(to + 8 * kWaves * n, y[n]);
        }
        if (wave == 0 && g == 0) a.part_ml[part * 32 + r32] = make_float2(top, sum);
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ many queries: K and V shared through LDS

// The descriptor of a buffer of `bytes` from p on, and 64 pieces of 16 bytes from it (this lane's: at voffset) into LDS from `to` on.  As
// builtins the compiler waits for all of them in front of any read of LDS; here the kernel waits by itself, once a block.  Nothing is
// written but LDS, and the wait (for everything that is out) stands before the barrier behind which it is read.
__device__ __forceinline__ u32x4 buffer_of(const void* p, uint32_t bytes) {
  const uint64_t at = (uint64_t)p;
  return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00020000u};
}
__device__ __forceinline__ void load_to_lds(const unsigned char* to, const u32x4& from, int voffset) {
  uint32_t m0;                           // (the compiler's own is put back)
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(lds_address(to)), "v"(voffset), "s"(from)
               : "memory");
}

// 2500 causal queries on 7000 keys, 32 heads of 128: 266 - 302 us by card and clock, 0.78 - 0.89 PFLOP/s of what the masks leave (a product of 8192^3 by the library: 1.23);
// matrix cores busy 51 %, vector units 49 % of the time, and the clock falls with both: a block of 64 keys went from 6100 clocks to 4200 as requests were
// spread between instructions, and from 2.76 us to 2.3 only.
// Eight tiles of 32 queries per workgroup, one a wave.  K and V of 64 keys (float: 32) at a time go from the pages straight into LDS, where they lie as in
// memory, so that every operand is 16 neighbouring bytes a lane.
// The two waves of a SIMD take turns: while one is at its matrix instructions (P V of the last block, Q K of this one) the other is at its exponentials.
// Time goes in half steps, each ended by a barrier: waves 0 - 3 have the products of block k in half step 2k and its softmax in 2k + 1, waves 4 - 7 one
// half step later.  In half step 2k waves 0 - 3 request V of block k between their products, waves 4 - 7 K of block k + 1 between their exponentials (whoever
// read their places before has passed a barrier since); they have to be there at the end of 2k + 1.
template <typename T, int D>
__global__ __launch_bounds__(512, 2) void pg_many_kernel(const AttendArgs a) {
  constexpr int E = 16 / sizeof(T), DT = D / 32, NF = D / (2 * E), NS = kPgUnit / (2 * E), kUnits = sizeof(T) == 2 ? 2 : 1;
  constexpr int kUnitBytes = kPgUnit * D * (int)sizeof(T), kOperand = kUnits * kUnitBytes, kPieces = kUnitBytes / 1024, kLoads = kUnits * kPieces / 4;
  constexpr int kRing = 4, kPerMm = sizeof(T) == 2 ? 1 : 4, kAll = (1 << kUnits) - 1;
  extern __shared__ __attribute__((aligned(16))) unsigned char plan_lds[];
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * 2 * kOperand];      // K, K, V, V
  __shared__ int range[kManyWaves][4];
  __shared__ uint32_t dropped_in[32];                   // blocks k % 1024 of which `clean` took something out
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, r32 = lane & 31;
  const int v_lane = (g * D + r32) * 16;
  const bool second = wave >= kManyWaves / 2;
  fetch_arguments(a);
  const Plan plan = make_plan<kManyWaves, 64 * kManyWaves>(a, plan_lds, 8.f, 0.06f);
  const int G = a.G;
  const size_t head_pitch = (size_t)D << a.page_log2;           // elements
  for (int round = 0; (int64_t)round * gridDim.x < plan.items; ++round) {
    // every other round backwards: the tiles of a masked prompt get shorter from item to item
    const int at_wg = round & 1 ? pg_backwards((int)blockIdx.x, (int)gridDim.x) : (int)blockIdx.x;
    const int item = round * gridDim.x + at_wg;
    if (item >= plan.items) continue;
    const Found found = find(plan, a.batch.batch, item);
    const int b = found.b;
    const PlanSeq s = found.seq;
    const Place at_item = place_of<kManyWaves>(a, found, item);
    const int hk = at_item.hk, split = at_item.split, tile = at_item.tile, splits = at_item.splits, R = s.m * G, sub = tile * kManyWaves + wave;
    const bool active = sub * 32 < R;
    const Queries q = queries_of(a, s, b, hk, active ? sub * 32 : tile * kManyWaves * 32, r32);
    u32x4 qf[NF];
    const T* qrow = (const T*)a.q + (int64_t)q.row * a.q_ld + q.head * D + g * E;
#pragma unroll
    for (int f = 0; f < NF; ++f) qf[f] = ld16(qrow + f * 2 * E);
    // keys that any wave sees, and that all of them see
    if (lane == 0) { range[wave][0] = q.all_lo; range[wave][1] = q.all_hi; range[wave][2] = q.both_lo; range[wave][3] = q.both_hi; }
    if (threadIdx.x < 32) dropped_in[threadIdx.x] = 0;
    __syncthreads();
    int lo = range[0][0], hi = range[0][1], in_lo = range[0][2], in_hi = range[0][3];
#pragma unroll
    for (int w = 1; w < kManyWaves; ++w) {
      lo = min(lo, range[w][0]);
      hi = max(hi, range[w][1]);
      in_lo = max(in_lo, range[w][2]);
      in_hi = min(in_hi, range[w][3]);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    in_lo = __builtin_amdgcn_readfirstlane(in_lo);
    in_hi = __builtin_amdgcn_readfirstlane(in_hi);
    int u0 = splits == 1 ? 0 : s.unit0 + split * plan.chunk, u1 = splits == 1 ? 0x7fffffff : u0 + plan.chunk;
    if (hi > 0) {
      u0 = max(u0, lo / kPgUnit);
      u1 = min(u1, (hi + kPgUnit - 1) / kPgUnit);
    } else u1 = u0;
    const int n_units = max(0, u1 - u0), n_blocks = (n_units + kUnits - 1) / kUnits;

    const int32_t* pages = a.batch.pages + (int64_t)b * a.batch.page_cols;
    // Of 64 units, one a lane: where it lies in the pools (bytes).  Waves 0 - 3 request V of block k, waves 4 - 7 K of block k + 1 (which they find first).
    uint32_t at_low = 0, at_high = 0;
    uint64_t have = 0;                        // which of them are there
    uint32_t flags = 0;                       // which units of the last blocks are there: kUnits bits at 2 (k % 16)
    auto there = [&](int k) __attribute__((always_inline)) { return (int)(flags >> (2 * (k & 15))) & kAll; };
    auto find_block = [&](int k) __attribute__((always_inline)) {
      const int first = k * kUnits & 63;
      if (first == 0) {
        const int unit = min(u0 + k * kUnits + lane, u1 - 1), page = pages[unit >> (a.page_log2 - 5)];
        const size_t at = (((size_t)page * a.Hkv + hk) * head_pitch + (size_t)(unit & ((1 << (a.page_log2 - 5)) - 1)) * kPgUnit * D) * sizeof(T);
        at_low = (uint32_t)at;
        at_high = (uint32_t)(at >> 32);
        have = __ballot(k * kUnits + lane < n_units && (unsigned)page < (unsigned)a.pages.n_pages);
        asm volatile("" : "+v"(at_low), "+v"(at_high));      // (the wait for the page numbers belongs here: behind the branch it would be one for all that is out, each time)
      }
      flags = (flags & ~(3u << (2 * (k & 15)))) | ((uint32_t)(have >> first) & kAll) << (2 * (k & 15));
    };
    // the j-th of a wave's kLoads pieces of a block; of a unit that is not there nothing is read (a buffer of no bytes)
    auto load = [&](const void* pool, int place, int k, int j) __attribute__((always_inline)) {
      const int u = j * 4 / kPieces, piece = j * 4 % kPieces + (wave & 3), l = (k * kUnits & 63) + u;
      const bool is = there(k) >> u & 1;
      const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_high, l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)at_low, l);
      load_to_lds(lds + (place + (k & 1)) * kOperand + u * kUnitBytes + piece * 1024, buffer_of((const char*)pool + (is ? off : 0) + piece * 1024, is ? 1024 : 0),
                  lane * 16);
    };
    auto nothing = [](int) {};
    auto requested = [&]() __attribute__((always_inline)) {       // everything this wave has requested is there (vmcnt(0))
      __builtin_amdgcn_s_waitcnt(0x70 | 0xf00);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto barrier = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };

    // V of a block of which a query of the workgroup does not see a key, once it is there: zeroed where none does, and where it is not
    // finite, so that the products need not look.  All waves; a barrier more.
    auto inside = [&](int k) __attribute__((always_inline)) {
      const int key0 = (u0 + k * kUnits) * kPgUnit;
      return there(k) == kAll && key0 >= in_lo && key0 + kUnits * kPgUnit <= in_hi;
    };
    auto clean = [&](int k) __attribute__((always_inline)) {
      if (inside(k)) return;
      const int key0 = (u0 + k * kUnits) * kPgUnit;
      u32x4* v = reinterpret_cast<u32x4*>(lds + (2 + (k & 1)) * kOperand);
      bool dropped = false;
      for (int i = threadIdx.x; i < kOperand / 16; i += 64 * kManyWaves) {
        const int u = i / (kUnitBytes / 16), key = key0 + u * kPgUnit + i % (kUnitBytes / 16) / D * E;
        u32x4 x = there(k) >> u & 1 ? keep_keys<T>(v[i], key, lo, hi) : u32x4{};
        dropped = drop_not_finite<T>(x) || dropped;
        v[i] = x;
      }
      if (dropped) atomicOr(&dropped_in[k / 32 % 32], 1u << (k & 31));
      __syncthreads();
    };

    f32x16 o[DT] = {}, acc[kUnits];
    u32x4 p[kUnits][NS];
    float ref = kFloor, l = 0.f;
    // One block's P V (the last block's) and Q K as a row of matrix instructions, operands through a ring of registers, the next ones requested right
    // behind the instruction that uses the last ones (the scheduler is told to keep that order).
    auto products = [&](auto with_pv, auto with_qk, int k, auto load) __attribute__((always_inline)) {
      constexpr int NV = with_pv ? kUnits * NS * DT : 0, N = NV + (with_qk ? kUnits * NF : 0);
      const unsigned char *kb = lds + (k & 1) * kOperand + lane * 16, *vb = lds + (2 + (~k & 1)) * kOperand + v_lane;
      u32x4 ring[kRing];
      auto read = [&](int i) __attribute__((always_inline)) {
        return *reinterpret_cast<const u32x4*>(i < NV ? vb + i / (NS * DT) * kUnitBytes + i / DT % NS * (2 * D * 16) + i % DT * 512
                                                      : kb + (i - NV) / NF * kUnitBytes + (i - NV) % NF * 1024);
      };
#pragma unroll
      for (int i = 0; i < kRing; ++i) ring[i] = read(i);
      __builtin_amdgcn_sched_group_barrier(0x100, kRing, 0);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        load(j);
#pragma unroll
        for (int i = j * (N / kLoads); i < (j + 1) * (N / kLoads); ++i) {
          if (i < NV) o[i % DT] = mm<T>(ring[i % kRing], p[i / (NS * DT)][i / DT % NS], o[i % DT]);
          else {
            const int u = (i - NV) / NF, f = (i - NV) % NF;
            acc[u] = mm<T>(ring[i % kRing], qf[f], f == 0 ? f32x16{} : acc[u]);
          }
          if (i + kRing < N) ring[i % kRing] = read(i + kRing);
        }
#pragma unroll
        for (int i = j * (N / kLoads); i < (j + 1) * (N / kLoads); ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, kPerMm, 0);
          if (i + kRing < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto softmax = [&](int k, auto load) __attribute__((always_inline)) {
      const int key0 = (u0 + k * kUnits) * kPgUnit;
      if (!(there(k) == kAll && key0 >= q.both_lo && key0 + kUnits * kPgUnit <= q.both_hi)) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const bool is = there(k) >> u & 1;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = key0 + u * kPgUnit + key_of<T>(i, g);
            acc[u][i] = is && key >= q.lo && key < q.hi ? acc[u][i] : -INFINITY;
          }
        }
      }
      float top = top_of(acc[0]);
#pragma unroll
      for (int u = 1; u < kUnits; ++u) top = fmaxf(top, top_of(acc[u]));
      raise<DT>(top, a.c2, ref, l, o);
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
#pragma unroll
        for (int j = u * (kLoads / kUnits); j < (u + 1) * (kLoads / kUnits); ++j) load(j);
        exps_unit<T>(acc[u], a.c2, ref, l, p[u]);
        __builtin_amdgcn_sched_barrier(0);
      }
      // (here and not behind the barrier)
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int i = 0; i < NS; ++i) asm volatile("" : "+v"(p[u][i]));
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    // the end of half step 2k or 2k + 1
    auto half = [&]() __attribute__((always_inline)) { barrier(); };
    auto full = [&](int k) __attribute__((always_inline)) {
      requested();
      barrier();
      clean(k);
    };

    if (n_blocks > 0) {
      if (!second) {
        auto load_v = [&](int k) { return [&, k](int j) __attribute__((always_inline)) { load(a.pages.v, 2, k, j); }; };
        auto step = [&](auto with_pv, int k) __attribute__((always_inline)) {
          find_block(k);
          if (active) products(with_pv, yes, k, load_v(k));
          else
            for (int j = 0; j < kLoads; ++j) load_v(k)(j);
          half();
          if (active) softmax(k, nothing);
          full(k);
        };
        barrier();
        step(no, 0);
        for (int k = 1; k < n_blocks; ++k) step(yes, k);
        if (active) products(yes, no, n_blocks, nothing);
        half();
      } else {
        auto load_k = [&](int k) { return [&, k](int j) __attribute__((always_inline)) { load(a.pages.k, 0, k, j); }; };
        auto load_all = [&](int k) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < kLoads; ++j) load_k(k)(j);
        };
        find_block(0);
        load_all(0);
        requested();
        barrier();
        find_block(1);
        load_all(1);
        half();
        if (active) products(no, yes, 0, nothing);
        full(0);
        find_block(2);
        if (active) softmax(0, load_k(2));
        else load_all(2);
        half();
        for (int k = 1; k < n_blocks; ++k) {
          if (active) products(yes, yes, k, nothing);
          full(k);
          find_block(k + 2);
          if (active) softmax(k, load_k(k + 2));
          else load_all(k + 2);
          half();
        }
        if (active) products(yes, no, n_blocks, nothing);
      }
    }

    // what `clean` took out, for the queries that see it (it can come last: a sum that has met infinity or NaN stays there)
    if (active && n_blocks > 0 && __builtin_expect(__ballot(dropped_in[lane & 31] != 0) != 0, 0)) {
#pragma unroll 1
      for (int k = 0; k < n_units; ++k) {
        const int unit = u0 + k, page = pages[unit >> (a.page_log2 - 5)], block = k / kUnits;
        if (!(dropped_in[block / 32 % 32] >> (block & 31) & 1) || (unsigned)page >= (unsigned)a.pages.n_pages) continue;
        add_not_finite<T, DT>((const T*)a.pages.v + ((size_t)page * a.Hkv + hk) * head_pitch + (size_t)(unit & ((1 << (a.page_log2 - 5)) - 1)) * kPgUnit * D,
                              unit * kPgUnit, q, o);
      }
    }
    l += __shfl_xor(l, 32, kWave);
    if (active && q.valid) {
      if (splits == 1) {
        const float inv = inverse_of(l);
        T* to = (T*)a.out + (int64_t)q.row * a.out_ld + q.head * D + 4 * g;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            store4<T>(to + 32 * dt + 2 * i, f32x4{o[dt][i] * inv, o[dt][i + 1] * inv, o[dt][i + 2] * inv, o[dt][i + 3] * inv});
        if (a.row_ml && g == 0) a.row_ml[(size_t)q.row * a.H + q.head] = make_float2(ref, inv);
      } else {
        const size_t part = (size_t)(found.split & 0xffffff) + ((size_t)hk * split_tiles<kManyWaves>(R, found.whole) + sub) * splits + split;
        float* to = a.part_o + (part * 32 + r32) * D + 4 * g;
        if (n_units > 0) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; i += 4) store4<float>(to + 32 * dt + 2 * i, f32x4{o[dt][i], o[dt][i + 1], o[dt][i + 2], o[dt][i + 3]});
        }
        if (g == 0) a.part_ml[part * 32 + r32] = make_float2(ref, l);
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ splits joined

// Groups of D / 4 lanes. Up to 8 splits: a group for each query, all of its splits requested at once; more: a workgroup for each query, its groups take
// the splits in turn, and their sums are added in order.  What a split that saw nothing of the query (sum 0) left is not used.  A launch of its own:
// 2.6 - 4 us for a token, 9 for 64 tiles of 256 queries in 4 splits (34 MB).
template <typename T, int D>
__global__ __launch_bounds__(256) void pg_join_kernel(const AttendArgs a) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kFew = 8, kEach = kPgMaxSplits / kGroups;
  __shared__ f32x4 sums[kGroups][kLanes];
  const int lane = threadIdx.x & 63, G = a.G, group = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
  for (int job = blockIdx.x;; job += gridDim.x) {
    int b = -1, before = 0, local = 0;
    int4 info = make_int4(0, 0, 0, 0);
    for (int b0 = 0; b0 < a.batch.batch && b < 0; b0 += 64) {
      const int4 mine = b0 + lane < a.batch.batch ? a.info[b0 + lane] : make_int4(1, 0, 0, 0);
      const int splits = mine.x & 255, n = splits > 1 ? a.Hkv * mine.y * (splits > kFew ? 32 : 32 / kGroups) : 0, end = scan_sum(n);
      const uint64_t past = __ballot(before + end > job);
      if (past) {
        const int at = (int)__builtin_ctzll(past);
        b = b0 + at;
        local = job - (before + __builtin_amdgcn_readlane(end - n, at));
        info = make_int4(__builtin_amdgcn_readlane(mine.x, at), __builtin_amdgcn_readlane(mine.y, at), __builtin_amdgcn_readlane(mine.z, at),
                         __builtin_amdgcn_readlane(mine.w, at));
      } else before += last_lane(end);
    }
    if (b < 0) return;
    const int splits = info.x & 255, per = splits > kFew ? 32 : 32 / kGroups;       // jobs of a tile
    const int hk = local / (per * info.y), sub = local / per % info.y;
    const size_t part = (size_t)(info.x >> 8) + ((size_t)hk * info.y + sub) * splits;
    const int at = splits > kFew ? local % 32 : local % per * kGroups + group, pair = sub * 32 + at;
    const bool valid = pair < info.w * G;
    const float2* ml = a.part_ml + part * 32 + (valid ? at : 0);
    const float* from = a.part_o + (part * 32 + (valid ? at : 0)) * D + d;
    float top = kFloor, sum = 0.f;
    f32x4 y = {};
    if (splits <= kFew) {
      f32x4 v[kFew];
      float2 m[kFew];
#pragma unroll
      for (int i = 0; i < kFew; ++i) {
        m[i] = i < splits ? ml[i * 32] : make_float2(kFloor, 0.f);
        v[i] = i < splits ? *reinterpret_cast<const f32x4*>(from + (size_t)i * 32 * D) : f32x4{};
      }
#pragma unroll
      for (int i = 0; i < kFew; ++i) top = fmaxf(top, m[i].x);
#pragma unroll
      for (int i = 0; i < kFew; ++i) {
        const float w = exp2_hw(m[i].x - top);
        sum += m[i].y * w;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] += m[i].y == 0.f ? 0.f : v[i][k] * w;
      }
    } else {
      f32x4 v[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int s = i * kGroups + group;
        v[i] = s < splits ? *reinterpret_cast<const f32x4*>(from + (size_t)s * 32 * D) : f32x4{};
      }
      const float2 m = lane < splits ? ml[lane * 32] : make_float2(kFloor, 0.f);
      top = wave_max(m.x);
      const float weight = exp2_hw(m.x - top);
      sum = wave_sum(m.y * weight);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int s = i * kGroups + group;
        const float w = __shfl(weight, s, kWave), saw = __shfl(m.y, s, kWave);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] += saw == 0.f ? 0.f : v[i][k] * w;
      }
      __syncthreads();                       // (the sums of the job before have been read)
      sums[group][d / 4] = y;
      __syncthreads();
      y = sums[0][d / 4];
#pragma unroll
      for (int i = 1; i < kGroups; ++i) y += sums[i][d / 4];
    }
    if (valid && (splits <= kFew || group == 0)) {
      const float inv = inverse_of(sum);
      const int r = info.z + pair / G, head = hk * G + pair % G;
      store4<T>((T*)a.out + (int64_t)r * a.out_ld + head * D + d, y * inv);
      if (a.row_ml && d == 0) a.row_ml[(size_t)r * a.H + head] = make_float2(top, inv);
    }
  }
}

// ------------------------------------------------------------------ the head average

// A workgroup takes 32 rows of a sequence and one or two units of its keys; its eight waves take the heads in turn and the waves' sums are added in order.
// Scores are computed again: kept ones would be H times the average's bytes, out and in.  Tiles of rows that read the same keys are neighbours on
// one XCD: blockIdx.x = (group of units / 8 * tiles + tile) * 8 + group % 8, tiles of 32 rows sequence after sequence.  4 sequences of 38 - 45 rows on 1823
// keys, 32 heads: 19 us (one round of workgroups: each wave's chain Q, K -> scores -> exponentials, four heads long; without the order by XCD 28).
template <typename T, int D> constexpr int kAvgUnits = D * (int)sizeof(T) > 256 ? 1 : 2;      // (float heads of 128 have registers for one)
template <typename T, int D>
__global__ __launch_bounds__(512, 2) void pg_average_kernel(const AttendArgs a, float* avg, int64_t avg_ld, int tiles, int wide) {
  constexpr int E = 16 / sizeof(T), NF = D / (2 * E), kW = 8, U = kAvgUnits<T, D>;
  __shared__ float sums[kW][32][33];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, r32 = lane & 31;
  const int at_tile = (int)(blockIdx.x / 8) % tiles, at_group = (int)(blockIdx.x / 8) / tiles * 8 + (int)(blockIdx.x % 8);
  // the sequence of this tile of rows
  int b = -1, tile = 0, before = 0;
  for (int b0 = 0; b0 < a.batch.batch && b < 0; b0 += 64) {
    const int s = b0 + lane;
    int n = 0;
    if (s < a.batch.batch) n = (pg_span(a.batch.row_start[s], a.batch.row_start[s + 1], a.batch.n_rows).m + 31) / 32;
    const int end = scan_sum(n);
    const uint64_t past = __ballot(before + end > at_tile);
    if (past) {
      const int at = (int)__builtin_ctzll(past);
      b = b0 + at;
      tile = at_tile - (before + __shfl(end - n, at, kWave));
    } else before += last_lane(end);
  }
  if (b < 0) return;
  const PgSpan span = pg_span(a.batch.row_start[b], a.batch.row_start[b + 1], a.batch.n_rows);
  const int row0 = span.row0, m = span.m;
  const int length = max(0, min(a.batch.length[b], a.batch.page_cols << a.page_log2));
  const int cols = (int)min((int64_t)length, avg_ld);
  const bool valid = tile * 32 + r32 < m;
  const int row = row0 + (valid ? tile * 32 + r32 : tile * 32);
  int lo, hi;
  visible(a, a.batch.at ? a.batch.at[row] : length - m + (row - row0), a.batch.origin ? max(0, a.batch.origin[b]) : 0, length, lo, hi);
  const int all_lo = reduce_min(lo), all_hi = reduce_max(hi), both_lo = reduce_max(lo), both_hi = reduce_min(hi);
  const int32_t* pages = a.batch.pages + (int64_t)b * a.batch.page_cols;
  const size_t head_pitch = (size_t)D << a.page_log2;
  const float share = 1.f / (float)a.H;
  for (int64_t u0 = (int64_t)at_group * U; u0 * kPgUnit < cols; u0 += (int64_t)wide * U) {
    size_t at[U];
    bool any[U];                         // a unit that is there, and that some row of the tile sees; others: zeros
    float total[U][16] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = (int)u0 + u, key0 = unit * kPgUnit;
      at[u] = 0;
      any[u] = key0 < cols && key0 < all_hi && key0 + kPgUnit > all_lo;
      if (any[u]) {
        const int page = pages[unit >> (a.page_log2 - 5)];
        any[u] = (unsigned)page < (unsigned)a.pages.n_pages;
        if (any[u]) at[u] = (size_t)page * a.Hkv * head_pitch + (size_t)(unit & ((1 << (a.page_log2 - 5)) - 1)) * kPgUnit * D;
      }
    }
    // the next head's operands are requested behind the products of this one
    u32x4 kr[U][NF], qr[NF];
    float2 ml;
    auto load = [&](int head) __attribute__((always_inline)) {
      const T* qrow = (const T*)a.q + (int64_t)row * a.q_ld + head * D + g * E;
      ml = a.row_ml[(size_t)row * a.H + head];
#pragma unroll
      for (int f = 0; f < NF; ++f) qr[f] = ld16(qrow + f * 2 * E);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const T* base = (const T*)a.pages.k + at[u] + (head / a.by_g) * head_pitch + (g * kPgUnit + r32) * E;
#pragma unroll
        for (int f = 0; f < NF; ++f)
          if (any[u]) kr[u][f] = ld16(base + 2 * f * kPgUnit * E);
      }
    };
    if (wave < a.H) load(wave);
    for (int head = wave; head < a.H; head += kW) {
      f32x16 acc[U] = {};
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (any[u])
#pragma unroll
          for (int f = 0; f < NF; ++f) acc[u] = mm<T>(kr[u][f], qr[f], acc[u]);
      const float2 now = ml;
      if (head + kW < a.H) load(head + kW);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!any[u]) continue;
        const int key0 = ((int)u0 + u) * kPgUnit;
        if (key0 >= both_lo && key0 + kPgUnit <= both_hi) {
#pragma unroll
          for (int i = 0; i < 16; ++i) total[u][i] = fmaf(exp2_hw(fmaf(acc[u][i], a.c2, -now.x)), now.y, total[u][i]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = key0 + key_of<T>(i, g);
            const float p = exp2_hw(fmaf(acc[u][i], a.c2, -now.x)) * now.y;
            total[u][i] += key >= lo && key < hi ? p : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key0 = ((int)u0 + u) * kPgUnit;
      if (key0 >= cols) break;
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[wave][r32][key_of<T>(i, g)] = total[u][i];
      __syncthreads();
      for (int c = threadIdx.x; c < 32 * 32; c += 64 * kW) {
        const int rr = c / 32, key = c % 32;
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) y += sums[w][rr][key];
        if (tile * 32 + rr < m && key0 + key < cols) avg[(int64_t)(row0 + tile * 32 + rr) * avg_ld + key0 + key] = y * share;
      }
      __syncthreads();
    }
  }
}

}  // namespace

constexpr int kMaxParts = 12288;       // 16.6 KB each with heads of 128

PgWorkspace pg_workspace(const PgShape& s, int max_rows, int max_batch) {
  PgWorkspace w{};
  if (max_rows <= 0) return w;
  const int64_t G = s.H / s.Hkv;
  w.parts = (int)std::min<int64_t>(kMaxParts, (max_rows * G / 32 + std::min(max_rows, max_batch)) * s.Hkv * kPgMaxSplits);
  auto take = [&](size_t bytes) {
    const size_t at = w.bytes;
    w.bytes += (bytes + 255) & ~(size_t)255;
    return at;
  };
  w.part_o = take((size_t)w.parts * 32 * s.D * 4);
  w.part_ml = take((size_t)w.parts * 32 * 8);
  w.row_ml = take((size_t)max_rows * s.H * 8);
  w.info = take((size_t)max_batch * 16);
  return w;
}

template <typename T, int D>
static hipError_t attention_d(const PgShape& s, AttendArgs a, const PgAttend& call, int cus, hipStream_t st) {
  const PgBatch& b = a.batch;
  // units of the longest cache that the page table can name
  const int64_t units = (int64_t)b.page_cols << (s.page_log2 - 5);
  // Short caches are not split: a second launch costs more than it saves (us, one token, 28 heads on 4: 200 keys 10.9, split 12.8; 600 keys 13.9 and 13.0).
  // Longer ones of bf16 neither, if workgroups of eight waves, one a compute unit, take all tiles at once: up to 768 keys, or 1536 where there are too many tiles
  // for many splits (one token, 28 heads on 4: 450 keys 11.6, split 12.1, 800 keys 12.0 and 12.0, 1023 keys 13.7 and 12.4; 100 rows, 32 heads: 600 keys 13.2
  // and 18.7, 1536 keys 18.0 and 22.2, 2040 keys 21.9 and 22.8; 200 rows, 12 heads of 64 on 2: 700 keys 10.5 and 13.2; float 4 heads of 64, 389 keys 17 and 16).
  const int64_t queries = (int64_t)b.n_rows * (s.H / s.Hkv), tiles = ((queries + 31) / 32 + std::min(b.n_rows, b.batch)) * s.Hkv;
  const bool small = units <= (sizeof(T) == 4 ? 2 : 3) * kFewWaves;
  const bool wide = !small && sizeof(T) == 2 && tiles <= cus && units <= (tiles > 64 ? 48 : 24) && b.batch <= 256;      // (there is LDS for the plan of 256)
  a.max_splits = small || wide ? 1 : (int)std::min<int64_t>(kPgMaxSplits, units / kFewWaves);
  hipError_t e = hipSuccess;
  const size_t lds = plan_bytes(b.batch);
  // Few products or many: each sequence goes by its own work, which only the device knows.  What the host knows: all together cannot have that much
  // work; or as many rows as sequences, single tokens (if they are not, the kernel for few queries takes them all).
  const double most = (double)b.n_rows * s.H * std::min((double)((int64_t)b.page_cols << s.page_log2), a.window > 0 ? 2.0 * a.window : 1e30);
  const bool few_only = most <= kMuch<T, D> || b.n_rows <= b.batch;
  const int parts = a.part_limit;
  a.much = few_only ? 3e38f : kMuch<T, D>;
  a.together = few_only || sizeof(T) == 4 || D == 64 ? 3e38f : 0.5f * kMuch<T, D>;
  a.part_limit = few_only ? parts : parts / 4;
  if constexpr (sizeof(T) == 2) {
    if (wide) hipLaunchKernelGGL((pg_few_kernel<T, D, 2 * kFewWaves>), dim3((unsigned)tiles), dim3(128 * kFewWaves), lds, st, a);
  }
  if (!wide) hipLaunchKernelGGL((pg_few_kernel<T, D, kFewWaves>), dim3(2 * cus), dim3(64 * kFewWaves), lds, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (!few_only) {
    a.part_first = parts / 4;
    a.part_limit = parts;
    hipLaunchKernelGGL((pg_many_kernel<T, D>), dim3(cus), dim3(64 * kManyWaves), lds, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.max_splits > 1) {
    // no more workgroups than jobs (a sequence's last tile counts whole), or than fill the chip
    const int64_t jobs = s.Hkv * (a.max_splits > 8 ? 32 : 4) * ((queries + 31) / 32 + std::min(b.n_rows, b.batch));
    hipLaunchKernelGGL((pg_join_kernel<T, D>), dim3((unsigned)std::min<int64_t>(8 * cus, jobs)), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (call.avg) {
    // groups of units: a multiple of 8, and no more than leave 2^22 workgroups in all
    const int64_t tiles = (int64_t)b.n_rows / 32 + std::min(b.n_rows, b.batch), cols = std::min<int64_t>(call.avg_ld, (int64_t)b.page_cols << s.page_log2);
    const int64_t groups = (cols + 32 * kAvgUnits<T, D> - 1) / (32 * kAvgUnits<T, D>);
    const int64_t wide = std::max<int64_t>(1, std::min((groups + 7) / 8, (1 << 22) / 8 / tiles)) * 8;
    hipLaunchKernelGGL((pg_average_kernel<T, D>), dim3((unsigned)(wide * tiles)), dim3(512), 0, st, a, call.avg, call.avg_ld, (int)tiles, (int)wide);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_pg_attention(const PgShape& s, const PgPages& pages, const PgBatch& batch, const PgAttend& call, const PgWorkspace& w, void* ws,
                               int cus, hipStream_t st) {
  AttendArgs a{};
  a.batch = batch;
  a.pages = pages;
  a.q = call.q;
  a.out = call.out;
  a.q_ld = call.q_ld;
  a.out_ld = call.out_ld;
  a.H = s.H;
  a.Hkv = s.Hkv;
  a.G = s.H / s.Hkv;
  a.by_hkv = div_by(s.Hkv);
  a.by_g = div_by(a.G);
  a.page_log2 = s.page_log2;
  a.block = call.block;
  a.window = call.window;
  a.c2 = call.scale * 1.44269504088896341f;
  a.part_first = 0;
  a.part_limit = w.parts;
  char* at = (char*)ws;
  a.part_o = (float*)(at + w.part_o);
  a.part_ml = (float2*)(at + w.part_ml);
  a.row_ml = call.avg ? (float2*)(at + w.row_ml) : nullptr;
  a.info = (int4*)(at + w.info);
  if (s.dtype == kF32) return s.D == 64 ? attention_d<float, 64>(s, a, call, cus, st) : attention_d<float, 128>(s, a, call, cus, st);
  return s.D == 64 ? attention_d<bf16, 64>(s, a, call, cus, st) : attention_d<bf16, 128>(s, a, call, cus, st);
}

}  // namespace d2c
