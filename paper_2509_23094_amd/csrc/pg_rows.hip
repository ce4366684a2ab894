// Rows on their way into a paged cache and out of it: rotation by positions of several axes, append, read (see include/d2c_pg.h).
//
// A wave takes (a part of) one row.  Its lanes form the row's angles, a pair each, in 64 bits: positions may be any 32-bit number, and of a product
// in 32 bits nothing would be left behind the revolutions.  Only the fraction of a revolution goes on, in two floats: the first through
// sincospi, the second as a first-order correction.  Then each lane turns 16 dimensions of a head at a time, in fp32, rounded once.
// All of it is bound by memory, or by one launch's chain (position -> angle -> row) where rows are few: 6075 rows of 4096, float in, bf16 out, 31.5 us (4.7 TB/s);
// a prompt of 2500 rows with q, k and v of 4096 each into its pages and k, v back 53.7 us (3.8 TB/s); one row 2.7 us; 64 rows of 64 sequences 3.4 and 2.6 us.
#include <algorithm>

#include "internal.h"
#include "pg.h"

namespace d2c {
namespace {

constexpr int kThreads = 256;

// eight neighbouring values as floats, and as T
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const bf16x8 v = __builtin_bit_cast(bf16x8, ld16(p));
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = __builtin_bit_cast(f32x4, ld16(p)), b = __builtin_bit_cast(f32x4, ld16(p + 4));
#pragma unroll
  for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (bf16)x[j];
  *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, v);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// Eight dimensions from d on of row t of a unit of K: one piece of 16 bytes (float: two); of V: eight single values
template <typename T> __device__ __forceinline__ void store_k(T* unit, int t, int d, const float (&x)[8]) {
  constexpr int E = 16 / sizeof(T);
  T* at = unit + (d / E) * (kPgUnit * E) + pg_slot<T>(t) * E;
  if constexpr (E == 8) store8(at, x);
  else {
    *reinterpret_cast<f32x4*>(at) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(at + kPgUnit * E) = f32x4{x[4], x[5], x[6], x[7]};
  }
}
template <typename T> __device__ __forceinline__ void load_k(const T* unit, int t, int d, float (&x)[8]) {
  constexpr int E = 16 / sizeof(T);
  const T* at = unit + (d / E) * (kPgUnit * E) + pg_slot<T>(t) * E;
  if constexpr (E == 8) load8(at, x);
  else {
    const f32x4 a = __builtin_bit_cast(f32x4, ld16(at)), b = __builtin_bit_cast(f32x4, ld16(at + kPgUnit * E));
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
  }
}
template <typename T> __device__ __forceinline__ T* v_place(T* unit, int D, int t, int d) {
  constexpr int E = 16 / sizeof(T);
  return unit + (t / E) * (D * E) + d * E + t % E;
}

// What 32 neighbouring packed rows are, a row a lane (both halves of the wave the same): see pg_row_at.
__device__ __forceinline__ PgRowAt rows_at(const PgBatch& b, int r0, int page_log2) {
  const int lane = threadIdx.x & 63, r = r0 + (lane & 31);
  int seq = 0, first = 0, next = 0, len = 0;
  bool found = false;
  for (int s0 = 0; s0 < b.batch && !__all(found); s0 += 64) {
    const int s = min(s0 + lane, b.batch - 1);
    const int lo = b.row_start[s], hi = b.row_start[s + 1], n = b.length[s];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const int behind = __popcll(__ballot(s0 + lane < b.batch && hi <= r0 + j));
      mine = (lane & 31) == j ? behind : mine;
    }
    const int f = __shfl(lo, min(mine, 63), 64), e = __shfl(hi, min(mine, 63), 64), l = __shfl(n, min(mine, 63), 64);
    if (!found) {
      seq += mine;
      found = mine < 64;
      first = f;
      next = e;
      len = l;
    }
  }
  PgRowAt a{-1, 0, 0, 0, 0};
  if (!found || seq >= b.batch || r >= b.n_rows || r < first || r >= next || first < 0 || next > b.n_rows) return a;
  a.seq = seq;
  a.first = first;
  a.count = next - first;
  a.length = max(0, min(len, b.page_cols << page_log2));
  a.index = b.at ? b.at[r] : a.length - a.count + (r - first);
  return a;
}

// 32 packed rows and their places in V, for tiles that turn rows into V's pieces (E rows of a dimension) and back through LDS: rows E of
// which fill a piece move as 16 bytes, the others value by value (2 bytes, which for a whole prompt of 2500 rows x 4096 took 58 us of 80).
struct ValueRows {
  size_t at;                     // of dimension 0, this lane's row
  uint32_t in, there, lead, rest;      // rows of a sequence; that have a place; first rows of whole pieces; that are in none of those
};
template <typename T, int D>
__device__ __forceinline__ ValueRows value_rows(const PgBatch& batch, int n_pages, int Hkv, int r0, int page_log2) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  const PgRowAt row = rows_at(batch, r0, page_log2);
  ValueRows v;
  int page = -1;
  if (row.seq >= 0 && row.index >= 0 && row.index < row.length) page = batch.pages[(int64_t)row.seq * batch.page_cols + (row.index >> page_log2)];
  const bool there = (unsigned)page < (unsigned)n_pages;
  const int in = row.index & ((1 << page_log2) - 1), t = in & (kPgUnit - 1);
  v.at = there ? (((size_t)page * Hkv) << page_log2) * D + (size_t)(in & ~(kPgUnit - 1)) * D + (t / E) * (D * E) + t % E : 0;
  v.in = (uint32_t)__ballot(row.seq >= 0);
  v.there = (uint32_t)__ballot(there);
  const int lo = (int)(uint32_t)v.at, hi = (int)(uint32_t)(v.at >> 32);
  bool lead = there && t % E == 0 && (lane & 31) + E <= 32;
#pragma unroll
  for (int k = 1; k < E; ++k) {
    const int l = __shfl(lo, (lane + k) & 63, 64), h = __shfl(hi, (lane + k) & 63, 64);
    lead = lead && (v.there >> ((lane + k) & 31) & 1) && h == hi && l == lo + k;
  }
  v.lead = (uint32_t)__ballot(lead);
  uint32_t whole = 0;
#pragma unroll
  for (int k = 0; k < E; ++k) whole |= v.lead << k;
  v.rest = v.there & ~whole;
  return v;
}
__device__ __forceinline__ size_t value_at(const ValueRows& v, int j) {
  return (size_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v.at, j) | (size_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v.at >> 32), j) << 32;
}
template <typename T, int D> constexpr int kTileBytes = 32 * (D + 16 / (int)sizeof(T)) * (int)sizeof(T);

struct RowsArgs {
  PgRotation rot;
  PgBatch batch;
  PgRows rows;
  PgPages pages;
  int n, parts, Hkv, page_log2;
  int v_tiles, v_heads;                  // workgroups in front that bring V in tiles (0: with the rows), kv heads of each
};

// Where dimension octets of chunk `sub` (16 dimensions of a head) lie, and its first pair (-1: not turned)
template <bool kNeighbours> __device__ __forceinline__ void chunk_of(int sub, int n_pairs, int& d0, int& d1, int& pair) {
  const bool turned = 8 * sub < n_pairs;
  pair = turned ? 8 * sub : -1;
  if (kNeighbours) {
    d0 = 16 * sub;
    d1 = d0 + 8;
  } else {
    d0 = turned ? 8 * sub : 16 * sub;
    d1 = turned ? n_pairs + 8 * sub : d0 + 8;
  }
}

// 32 rows of V into their pages, v_heads kv heads of them
template <typename TS, typename T, int D> __device__ __forceinline__ void put_values(const RowsArgs& a, T* tile) {
  constexpr int E = 16 / sizeof(T), kPitch = D + E;
  const int groups = (a.n + 31) / 32, r0 = (int)blockIdx.x % groups * 32, h0 = (int)blockIdx.x / groups * a.v_heads;
  const ValueRows v = value_rows<T, D>(a.batch, a.pages.n_pages, a.Hkv, r0, a.page_log2);
  if (v.there == 0) return;
  const int d = threadIdx.x % D;
  for (int h = h0; h < min(a.Hkv, h0 + a.v_heads); ++h) {
    T* out = (T*)a.pages.v + (((size_t)h * D) << a.page_log2) + (size_t)d * E;
    for (int c = threadIdx.x; c < 32 * (D / 8); c += kThreads) {
      const int j = c / (D / 8), at = c % (D / 8) * 8;
      if (v.there >> j & 1) {
        float x[8];
        load8((const TS*)a.rows.v + (int64_t)(r0 + j) * a.rows.v_ld + h * D + at, x);
        store8(tile + j * kPitch + at, x);
      }
    }
    __syncthreads();
    int i = threadIdx.x / D;                   // (whole waves: D is 64 or 128)
    for (uint32_t m = v.lead; m; m &= m - 1, --i) {
      if (i % (kThreads / D)) continue;
      const int j = __builtin_ctz(m);
      union { T x[E]; u32x4 raw; } w;
#pragma unroll
      for (int k = 0; k < E; ++k) w.x[k] = tile[(j + k) * kPitch + d];
      *reinterpret_cast<u32x4*>(out + value_at(v, j)) = w.raw;
    }
    i = threadIdx.x / D;
    for (uint32_t m = v.rest; m; m &= m - 1, --i) {
      if (i % (kThreads / D)) continue;
      const int j = __builtin_ctz(m);
      out[value_at(v, j)] = tile[j * kPitch + d];
    }
    __syncthreads();
  }
}

// Workgroup wg of `count`, every 256 of them in another order: workgroups go round the 8 XCDs, and those of one XCD take neighbouring rows, because 8 rows'
// pieces of K share a line that should go through one L2 (a prompt of 2500 rows into its pages and back 72 us without, 66 with it in the append, 60 in both).
__device__ __forceinline__ int by_xcd(int wg, int count) {
  const int j = wg & 255;
  return wg - j + 256 <= count ? wg - j + (j & 7) * 32 + (j >> 3) : wg;
}

template <typename TS, typename T, int D, bool kNeighbours>
__global__ __launch_bounds__(kThreads) void pg_rows_kernel(const RowsArgs a) {
  __shared__ float2 table[kThreads / 64][64];
  __shared__ __attribute__((aligned(16))) unsigned char tile_lds[kTileBytes<T, D>];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < a.v_tiles) {
    put_values<TS, T, D>(a, reinterpret_cast<T*>(tile_lds));
    return;
  }
  const int wg = (int)blockIdx.x - a.v_tiles;
  const int64_t id = (int64_t)(a.rows.k ? by_xcd(wg, (int)gridDim.x - a.v_tiles) : wg) * (kThreads / 64) + wave;
  const int r = (int)(id / a.parts), part = (int)(id % a.parts);
  if (r >= a.n) return;
  PgRowAt row{0, 0, 0, 0, 0};
  if (a.batch.batch > 0) {
    row = pg_row_at(a.batch, r, a.page_log2);
    if (row.seq < 0) return;
  }
  float2* cs = table[wave];
  const int n_pairs = a.rot.n_pairs;
  if (lane < n_pairs) {
    const int pos = a.rows.pos ? a.rows.pos[(int64_t)a.rot.axis[lane] * a.n + r] : row.index;
    const double rev = (double)pos * a.rot.turns[lane];
    const double rest = rev - rint(rev);
    const float hi = (float)rest, lo = (float)(rest - (double)hi) * 6.2831853071795865f;
    float s, c;
    sincospif(2.f * hi, &s, &c);
    cs[lane] = make_float2(fmaf(-s, lo, c), fmaf(c, lo, s) * a.rows.sign);
  }
  // the row's place in the cache
  T *ku = nullptr, *vu = nullptr;
  int t = 0;
  if (row.index >= 0 && row.index < row.length) {
    const int page = a.batch.pages[(int64_t)row.seq * a.batch.page_cols + (row.index >> a.page_log2)];
    if ((unsigned)page < (unsigned)a.pages.n_pages) {
      const int in = row.index & ((1 << a.page_log2) - 1);
      const size_t at = (((size_t)page * a.Hkv) << a.page_log2) * D + (size_t)(in & ~(kPgUnit - 1)) * D;
      t = in & (kPgUnit - 1);
      ku = (T*)a.pages.k + at;
      vu = (T*)a.pages.v + at;
    }
  }
  const size_t head_pitch = (size_t)D << a.page_log2;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the table is this wave's own
  __builtin_amdgcn_wave_barrier();

  constexpr int kSub = D / 16;
  const int nq = a.rows.q ? a.rows.q_heads * kSub : 0, nk = a.rows.k ? a.Hkv * kSub : 0, total = nq + (a.v_tiles ? nk : 2 * nk);
  const int per = ((total + 63) / 64 + a.parts - 1) / a.parts * 64;
  const int end = min(total, (part + 1) * per);
  for (int c = part * per + lane; c < end; c += 64) {
    const int kind = c < nq ? 0 : c < nq + nk ? 1 : 2;                  // q, k, v
    const int local = c - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk), head = local / kSub, sub = local % kSub;
    if (kind != 0 && !ku) continue;
    int d0 = 16 * sub, d1 = d0 + 8, pair = -1;
    if (kind != 2) chunk_of<kNeighbours>(sub, n_pairs, d0, d1, pair);
    const TS* src = kind == 0 ? (const TS*)a.rows.q + (int64_t)r * a.rows.q_ld : kind == 1 ? (const TS*)a.rows.k + (int64_t)r * a.rows.k_ld
                                                                                         : (const TS*)a.rows.v + (int64_t)r * a.rows.v_ld;
    float x[8], y[8];
    load8(src + head * D + d0, x);
    load8(src + head * D + d1, y);
    if (pair >= 0) {
      float2 w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = cs[pair + j];
      if constexpr (kNeighbours) {
        // pairs (x0, x1) .. (x6, x7), (y0, y1) ..
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float a0 = x[2 * j], b0 = x[2 * j + 1], a1 = y[2 * j], b1 = y[2 * j + 1];
          x[2 * j] = a0 * w[j].x - b0 * w[j].y;
          x[2 * j + 1] = b0 * w[j].x + a0 * w[j].y;
          y[2 * j] = a1 * w[4 + j].x - b1 * w[4 + j].y;
          y[2 * j + 1] = b1 * w[4 + j].x + a1 * w[4 + j].y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[j], q = y[j];
          x[j] = p * w[j].x - q * w[j].y;
          y[j] = q * w[j].x + p * w[j].y;
        }
      }
    }
    if (kind == 0) {
      T* to = (T*)a.rows.q_out + (int64_t)r * a.rows.q_out_ld + head * D;
      store8(to + d0, x);
      store8(to + d1, y);
    } else if (kind == 1) {
      store_k<T>(ku + head * head_pitch, t, d0, x);
      store_k<T>(ku + head * head_pitch, t, d1, y);
    } else {
      T* to = v_place<T>(vu + head * head_pitch, D, t, d0);
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j * (16 / sizeof(T))] = from_f32<T>(x[j]);
#pragma unroll
      for (int j = 0; j < 8; ++j) to[(8 + j) * (16 / sizeof(T))] = from_f32<T>(y[j]);
    }
  }
}

struct ReadArgs {
  PgBatch batch;
  PgPages pages;
  void *out_k, *out_v;
  int64_t k_ld, v_ld;
  int parts, Hkv, page_log2;
  int v_tiles, v_heads;                  // as above
};

// 32 rows of V from their pages
template <typename T, int D> __device__ __forceinline__ void get_values(const ReadArgs& a, T* tile) {
  constexpr int E = 16 / sizeof(T), kPitch = D + E;
  const int groups = (a.batch.n_rows + 31) / 32, r0 = (int)blockIdx.x % groups * 32, h0 = (int)blockIdx.x / groups * a.v_heads;
  const ValueRows v = value_rows<T, D>(a.batch, a.pages.n_pages, a.Hkv, r0, a.page_log2);
  if (v.in == 0) return;
  const int d = threadIdx.x % D;
  for (int h = h0; h < min(a.Hkv, h0 + a.v_heads); ++h) {
    const T* from = (const T*)a.pages.v + (((size_t)h * D) << a.page_log2) + (size_t)d * E;
    int i = threadIdx.x / D;
    for (uint32_t m = v.lead; m; m &= m - 1, --i) {
      if (i % (kThreads / D)) continue;
      const int j = __builtin_ctz(m);
      union { T x[E]; u32x4 raw; } w;
      w.raw = ld16(from + value_at(v, j));
#pragma unroll
      for (int k = 0; k < E; ++k) tile[(j + k) * kPitch + d] = w.x[k];
    }
    i = threadIdx.x / D;
    for (uint32_t m = v.rest; m; m &= m - 1, --i) {
      if (i % (kThreads / D)) continue;
      const int j = __builtin_ctz(m);
      tile[j * kPitch + d] = from[value_at(v, j)];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * (D / 8); c += kThreads) {
      const int j = c / (D / 8), at = c % (D / 8) * 8;
      if (v.in >> j & 1) {
        float x[8] = {};
        if (v.there >> j & 1) load8(tile + j * kPitch + at, x);
        store8((T*)a.out_v + (int64_t)(r0 + j) * a.v_ld + h * D + at, x);
      }
    }
    __syncthreads();
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pg_read_kernel(const ReadArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char tile_lds[kTileBytes<T, D>];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < a.v_tiles) {
    get_values<T, D>(a, reinterpret_cast<T*>(tile_lds));
    return;
  }
  const int64_t id = (int64_t)by_xcd((int)blockIdx.x - a.v_tiles, (int)gridDim.x - a.v_tiles) * (kThreads / 64) + wave;
  const int r = (int)(id / a.parts), part = (int)(id % a.parts);
  if (r >= a.batch.n_rows) return;
  const PgRowAt row = pg_row_at(a.batch, r, a.page_log2);
  if (row.seq < 0) return;
  int page = -1;
  if (row.index >= 0 && row.index < row.length) page = a.batch.pages[(int64_t)row.seq * a.batch.page_cols + (row.index >> a.page_log2)];
  const bool there = (unsigned)page < (unsigned)a.pages.n_pages;
  const int in = row.index & ((1 << a.page_log2) - 1), t = in & (kPgUnit - 1);
  const size_t at = there ? (((size_t)page * a.Hkv) << a.page_log2) * D + (size_t)(in & ~(kPgUnit - 1)) * D : 0;
  const size_t head_pitch = (size_t)D << a.page_log2;
  constexpr int kOct = D / 8, E = 16 / sizeof(T);
  const int nk = a.out_k ? a.Hkv * kOct : 0, total = nk + (a.out_v && !a.v_tiles ? a.Hkv * kOct : 0);
  const int per = ((total + 63) / 64 + a.parts - 1) / a.parts * 64;
  const int end = min(total, (part + 1) * per);
  for (int c = part * per + lane; c < end; c += 64) {
    const bool is_k = c < nk;
    const int local = is_k ? c : c - nk, head = local / kOct, d = local % kOct * 8;
    float x[8] = {};
    if (there) {
      if (is_k) load_k<T>((const T*)a.pages.k + at + head * head_pitch, t, d, x);
      else {
        const T* from = v_place<const T>((const T*)a.pages.v + at + head * head_pitch, D, t, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = to_f32(from[j * E]);
      }
    }
    store8((is_k ? (T*)a.out_k + (int64_t)r * a.k_ld : (T*)a.out_v + (int64_t)r * a.v_ld) + head * D + d, x);
  }
}

// Waves for each row, so that there are 8192 in all: eight a SIMD, for a load that is out has to cover 2 us of latency (6075 rows of 4096 32 us, with 2048 34; a
// prompt of 2500 rows into its pages and back 62 us, with 2048 70, with 16384 68, each before V's workgroups took four heads)
int parts_for(int n, int chunks) { return std::max(1, std::min((chunks + 63) / 64, (8192 + n - 1) / n)); }
// V in tiles of 32 rows and v_heads kv heads: how many workgroups, 0 where rows bring their V themselves.  Tiles pay where sequences have several rows
// (whole pieces), and from 2^18 values on.  Append and read, us, by rows and by tiles: one sequence, 32 kv heads of 128: 64 rows 12.0 and 11.1,
// 256 rows 24.5 and 15.3, 2048 rows 95 and 54; 4 kv heads: 256 rows 9.3 and 10.8, 512 rows 11.6 and 11.5, 1024 rows 15.6 and 13.5; 64 sequences
// of one row, 32 kv heads: 13.6 and 16.5, 1000 of them 73 and 87.  Up to four heads a workgroup, so that a row is read 1 KB at a time: 60 -> 54 us for 2500 rows
// (two 56.5, six 53.5; 8 sequences of 300 rows 54, with two 51).
int value_tiles(int n, int batch, int Hkv, int D, int& v_heads) {
  v_heads = 1;
  if (n / 8 < batch || (int64_t)n * Hkv * D < 1 << 18) return 0;
  const int64_t groups = (n + 31) / 32;
  v_heads = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(Hkv, 4), groups * Hkv / 512));
  return (int)(groups * ((Hkv + v_heads - 1) / v_heads));
}

template <typename TS, typename T, int D>
hipError_t rows_d(const RowsArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.v_tiles + ((int64_t)a.n * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
  if (a.rot.pairing) hipLaunchKernelGGL((pg_rows_kernel<TS, T, D, true>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((pg_rows_kernel<TS, T, D, false>), grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}
template <typename TS, typename T>
hipError_t rows_t(int D, const RowsArgs& a, hipStream_t st) {
  return D == 64 ? rows_d<TS, T, 64>(a, st) : rows_d<TS, T, 128>(a, st);
}

}  // namespace

hipError_t launch_pg_rows(const PgShape& s, const PgRotation& rot, const PgPages& pages, const PgBatch* batch, int n, const PgRows& rows,
                          hipStream_t st) {
  RowsArgs a{};
  a.rot = rot;
  if (batch) a.batch = *batch;
  a.rows = rows;
  a.pages = pages;
  a.n = n;
  a.Hkv = s.Hkv;
  a.page_log2 = s.page_log2;
  a.v_tiles = rows.v ? value_tiles(n, batch->batch, s.Hkv, s.D, a.v_heads) : 0;
  a.parts = parts_for(n, ((rows.q ? rows.q_heads : 0) + (rows.k ? s.Hkv : 0) + (rows.v && !a.v_tiles ? s.Hkv : 0)) * (s.D / 16));
  const bool from_f32 = rows.src_dtype == kF32;
  if (s.dtype == kF32) return rows_t<float, float>(s.D, a, st);
  return from_f32 ? rows_t<float, bf16>(s.D, a, st) : rows_t<bf16, bf16>(s.D, a, st);
}

hipError_t launch_pg_read(const PgShape& s, const PgPages& pages, const PgBatch& batch, void* out_k, int64_t k_ld, void* out_v, int64_t v_ld,
                          hipStream_t st) {
  ReadArgs a{batch, pages, out_k, out_v, k_ld, v_ld, 1, s.Hkv, s.page_log2, 0, 1};
  if (out_v) a.v_tiles = value_tiles(batch.n_rows, batch.batch, s.Hkv, s.D, a.v_heads);
  const int n_rest = (out_k != nullptr) + (out_v != nullptr && !a.v_tiles);
  a.parts = parts_for(batch.n_rows, n_rest * s.Hkv * (s.D / 8));
  const dim3 grid((unsigned)(a.v_tiles + (n_rest ? ((int64_t)batch.n_rows * a.parts + kThreads / 64 - 1) / (kThreads / 64) : 0)));
  if (s.dtype == kF32) {
    if (s.D == 64) hipLaunchKernelGGL((pg_read_kernel<float, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((pg_read_kernel<float, 128>), grid, dim3(kThreads), 0, st, a);
  } else {
    if (s.D == 64) hipLaunchKernelGGL((pg_read_kernel<bf16, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((pg_read_kernel<bf16, 128>), grid, dim3(kThreads), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace d2c
