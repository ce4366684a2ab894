// Rows on their way into a paged cache and out of it: rotation by positions of several axes, append, read (see include/d2c_pg.h).
//
// A wave takes (a part of) one row.  Its lanes form the row's angles, a pair each, in 64 bits: positions may be any 32-bit number, and of a product
// in 32 bits nothing would be left behind the revolutions.  Only the fraction of a revolution goes on, in two floats: the first through
// sincospi, the second as a first-order correction.  Then each lane turns 16 dimensions of a head at a time, in fp32, rounded once.
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

struct RowsArgs {
  PgRotation rot;
  PgBatch batch;
  PgRows rows;
  PgPages pages;
  int n, parts, H, Hkv, page_log2;
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

template <typename TS, typename T, int D, bool kNeighbours>
__global__ __launch_bounds__(kThreads) void pg_rows_kernel(const RowsArgs a) {
  __shared__ float2 table[kThreads / 64][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + wave;
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
  const int nq = a.rows.q ? a.rows.q_heads * kSub : 0, nk = a.rows.k ? a.Hkv * kSub : 0, total = nq + 2 * nk;
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
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pg_read_kernel(const ReadArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + wave;
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
  const int nk = a.out_k ? a.Hkv * kOct : 0, total = nk + (a.out_v ? a.Hkv * kOct : 0);
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

// A wave for each row, several where there are few: 2048 waves give each SIMD of the chip two
int parts_for(int n, int chunks) { return std::max(1, std::min((chunks + 63) / 64, (2048 + n - 1) / n)); }

template <typename TS, typename T, int D>
hipError_t rows_d(const RowsArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.n * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
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
  a.H = s.H;
  a.Hkv = s.Hkv;
  a.page_log2 = s.page_log2;
  a.parts = parts_for(n, ((rows.q ? rows.q_heads : 0) + (rows.k ? 2 * s.Hkv : 0)) * (s.D / 16));
  const bool from_f32 = rows.src_dtype == kF32;
  if (s.dtype == kF32) return rows_t<float, float>(s.D, a, st);
  return from_f32 ? rows_t<float, bf16>(s.D, a, st) : rows_t<bf16, bf16>(s.D, a, st);
}

hipError_t launch_pg_read(const PgShape& s, const PgPages& pages, const PgBatch& batch, void* out_k, int64_t k_ld, void* out_v, int64_t v_ld,
                          hipStream_t st) {
  ReadArgs a{batch, pages, out_k, out_v, k_ld, v_ld, 1, s.Hkv, s.page_log2};
  a.parts = parts_for(batch.n_rows, ((out_k != nullptr) + (out_v != nullptr)) * s.Hkv * (s.D / 8));
  const dim3 grid((unsigned)(((int64_t)batch.n_rows * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
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
