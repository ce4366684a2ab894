// The 8-bit K/V cache apart from its attention: refreshed rows in, rows out as values, attention weight summed, rows kept and
// the cache compacted.  All of it moves bytes: one pass over the codes and rows concerned, 16 bytes per access.
#include <algorithm>
#include <type_traits>

#include "q8.h"

namespace d2c {
namespace {

// One block of one kv head: 64 * D codes.  K pieces of 16 bytes: 16 dimensions of a row; V pieces: four dimensions of four rows.
template <int D> struct Pieces {
  static constexpr int kCount = kQ8Rows * D / 16;
  static constexpr int kPerThread = kCount / 256;
  // K: consecutive threads take the pieces of one row (256 bytes of bf16), then the next row
  __device__ static int k_row(int p) { return p / (D / 16); }
  __device__ static int k_dim(int p) { return p % (D / 16) * 16; }
  __device__ static int k_at(int p) { return k_dim(p) * kQ8Rows + k_row(p) * 16; }
  // V: consecutive threads take neighbouring dimensions of the same four rows: addresses are consecutive
  __device__ static int v_row(int p) { return p / (D / 4) * 4; }
  __device__ static int v_dim(int p) { return p % (D / 4) * 4; }
  __device__ static int v_at(int p) { return p * 16; }
};

struct UpdateArgs {
  Q8Update c[kQ8Launch];
};

constexpr int kScan = 1024;                  // so many indices are compared with a block's range each

// Number of idx entries below `limit`, by all 256 threads together (idx ascending; in bounds whatever it holds).
__device__ int lower_bound_wide(const int32_t* idx, int m, int limit) {
  const int step = (m + 255) / 256, t = threadIdx.x;
  const int c = __syncthreads_count((int64_t)t * step < m && idx[(int64_t)t * step] < limit);
  int lo = max(0, c - 1) * step, n = 0;
  for (int i = 0; i < step; i += 256) {
    const int at = lo + i + t;
    n += __syncthreads_count(i + t < step && at < m && idx[at] < limit);
  }
  return lo + n;
}

// A workgroup per (block, kv head, K or V, sequence).  Its refreshed rows are found first: blocks are counted from the first refreshed
// one where the rows are consecutive or many; few scattered rows get a workgroup each, of which the first of a block's does the block.
// Rows and, where the scale moves, the old codes are then read once and the codes written once.
// What bounds it: bytes for a whole prompt (2500 rows of 32 heads of 128, bf16: 18-21 us, 61 MB), the chain index -> rows -> maximum -> codes for a
// decode step (45 rows among 1823: 8.6 us where all fit their blocks' scales; 16.9 where the scale of every block they touch grows,
// which is then read and written whole).
template <typename T, int D>
__global__ __launch_bounds__(256) void q8_update_kernel(UpdateArgs args, int Hkv) {
  using P = Pieces<D>;
  const Q8Update c = args.c[blockIdx.z];
  const int h = blockIdx.y >> 1, is_v = blockIdx.y & 1, tid = threadIdx.x, slot = blockIdx.x;
  const int n_blocks = (c.L + kQ8Rows - 1) / kQ8Rows;
  __shared__ int row_of[kQ8Rows], near[kQ8Rows + 1];
  __shared__ float wave_amax[4];
  int b;
  if (tid < kQ8Rows) row_of[tid] = -1;
  if (!c.idx) {
    const int first = c.L - c.m;
    b = first / kQ8Rows + slot;
    if (b >= n_blocks) return;
    __syncthreads();
    const int pos = b * kQ8Rows + tid;
    if (tid < kQ8Rows && pos >= first && pos < c.L) row_of[tid] = pos - first;
  } else {
    if (c.m < n_blocks) {                       // a slot is a row; near: its index behind the one before
      if (slot >= c.m) return;
      if (tid <= kQ8Rows) near[tid] = c.idx[min(max(slot - 1 + tid, 0), c.m - 1)];
      __syncthreads();
      const int pos = near[1];
      if (pos < 0 || pos >= c.L) return;
      b = pos / kQ8Rows;
      if (slot > 0 && (near[0] >> 6) == b) return;
    } else {                                    // a slot is a block
      b = slot;
      if (b >= n_blocks) return;
    }
    auto take = [&](int i, int pos) {
      if (i < c.m && pos >= 0 && pos < c.L && pos / kQ8Rows == b) atomicMax(&row_of[pos % kQ8Rows], i);
    };
    if (c.m < n_blocks) {
      if (tid < kQ8Rows) take(slot + tid, near[1 + tid]);
    } else if (c.m <= kScan) {                  // looked at one and all: one latency instead of the search's three
      int pos[kScan / 256];
#pragma unroll
      for (int i = 0; i < kScan / 256; ++i) pos[i] = c.idx[min(tid + 256 * i, c.m - 1)];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kScan / 256; ++i) take(tid + 256 * i, pos[i]);
    } else {
      // as many indices as rows: index i is i, unless some are left out -- which the two on either side of the place tell (2500
      // rows, updated and read: 33.8 us, with the search always 35.2)
      const int start = b * kQ8Rows;
      bool found = false;
      if (c.m == c.L) {
        if (tid <= kQ8Rows) near[tid] = c.idx[min(max(start - 1 + tid, 0), c.m - 1)];
        __syncthreads();
        found = (start == 0 || near[0] < start) && near[1] >= start;
        if (found && tid < kQ8Rows) take(start + tid, near[1 + tid]);
      }
      if (!found) {
        const int lo = lower_bound_wide(c.idx, c.m, start);
        if (tid < kQ8Rows) take(lo + tid, c.idx[min(lo + tid, c.m - 1)]);
      }
    }
  }
  __syncthreads();
  const uint64_t fresh = __ballot(row_of[tid & 63] >= 0);
  if (fresh == 0) return;
  const int valid = min(kQ8Rows, c.L - b * kQ8Rows);
  const bool whole = __popcll(fresh) == valid;

  const T* rows = (const T*)(is_v ? c.new_v : c.new_k) + (size_t)h * D;
  const size_t pitch = (size_t)Hkv * D;
  const size_t base = ((size_t)b * Hkv + h) * kQ8Rows * D;
  uint8_t* codes = (is_v ? c.cache.v : c.cache.k) + base;
  float* scale = (is_v ? c.cache.vs : c.cache.ks) + (size_t)b * Hkv + h;
  const float s_old = *scale;

  // (rows that are not there are read as the first one and set to 0: loads under a condition would come one after the other)
  float x[P::kPerThread][16];
#pragma unroll
  for (int i = 0; i < P::kPerThread; ++i) {
    const int p = tid + 256 * i;
    if (is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
        q8_load4(rows + max(row_of[P::v_row(p) + j], 0) * pitch + P::v_dim(p), y);
#pragma unroll
        for (int d = 0; d < 4; ++d) x[i][4 * d + j] = y[d];                  // in the order of the piece's bytes
      }
    } else {
      const T* from = rows + max(row_of[P::k_row(p)], 0) * pitch + P::k_dim(p);
      float y[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        q8_load8(from + 8 * h, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][8 * h + j] = y[j];
      }
    }
  }
  // which rows of a piece are new: V its four rows, K all four bits alike; a V piece that stays in part is read now
  uint32_t is_new[P::kPerThread];
  u32x4 was[P::kPerThread];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < P::kPerThread; ++i) {
    const int p = tid + 256 * i;
    is_new[i] = is_v ? (uint32_t)(fresh >> P::v_row(p)) & 15u : (fresh >> P::k_row(p) & 1) ? 15u : 0u;
    was[i] = u32x4{0, 0, 0, 0};
    if (is_new[i] != 0 && is_new[i] != 15u) was[i] = ld16(codes + P::v_at(p));
  }
#pragma unroll
  for (int i = 0; i < P::kPerThread; ++i) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (!(is_new[i] >> (j & 3) & 1u)) x[i][j] = 0.f;
      const float a = fabsf(x[i][j]);
      amax = fmaxf(amax, a <= 3.402823466e38f ? a : 0.f);
    }
  }
  amax = wave_max(amax);
  if ((tid & 63) == 0) wave_amax[tid >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(wave_amax[0], wave_amax[1]), fmaxf(wave_amax[2], wave_amax[3]));
  const float want = q8_scale(amax);
  const float s = whole ? want : want > s_old ? fmaxf(want, s_old * 1.25f) : s_old;
  const bool moved = !whole && s != s_old;
  const float inv = q8_inverse(s), ratio = s_old * inv;
#pragma unroll
  for (int i = 0; i < P::kPerThread; ++i) {
    const int p = tid + 256 * i;
    if (is_new[i] == 0 && !moved) continue;
    u32x4* at = reinterpret_cast<u32x4*>(codes + (is_v ? P::v_at(p) : P::k_at(p)));
    u32x4 w = was[i];
    if (is_new[i] == 0) w = *at;
    uint32_t byte[16];
    q8_bytes16(x[i], s, inv, byte);
    const uint32_t keep = (is_new[i] & 1u ? 0u : 0xffu) | (is_new[i] & 2u ? 0u : 0xff00u) | (is_new[i] & 4u ? 0u : 0xff0000u) | (is_new[i] & 8u ? 0u : 0xff000000u);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t old = w[d];
      if (moved) old = q8_reword(old, s_old, s, inv, ratio);
      w[d] = (q8_pack(byte[4 * d], byte[4 * d + 1], byte[4 * d + 2], byte[4 * d + 3]) & ~keep) | (old & keep);
    }
    *at = w;
  }
  if (tid == 0 && s != s_old) *scale = s;      // every thread has read the old one before the barrier above
}

// A thread per (row, four dimensions of a kv head).  A workgroup's rows are neighbours, so that the four rows of a V piece, and the
// pieces of K in one line, come from the L1.
// What bounds it: bytes; 2500 rows of 32 heads of 128, bf16: 13.6 us, 61 MB.
template <typename T, int D>
__global__ __launch_bounds__(256) void q8_read_kernel(Q8CachePtr c, int L, const int32_t* idx, int n, int Hkv, T* out_k, T* out_v) {
  const int r = blockIdx.x * (1024 / D) + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4, h = blockIdx.y;
  if (r >= n) return;
  const int pos = idx ? idx[r] : r;
  float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (pos >= 0 && pos < L) {
    const int t = pos % kQ8Rows;
    const size_t g = (size_t)(pos / kQ8Rows) * Hkv + h, base = g * kQ8Rows * D;
    if (out_k) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(c.k + base + d / 16 * 1024 + t * 16 + d % 16);
      const float s = c.ks[g];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = (float)q8_code_of(w, j) * s;
    }
    if (out_v) {
      const u32x4 w = ld16(c.v + base + t / 4 * 4 * D + d * 4);
      const float s = c.vs[g];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (float)q8_code_of(w[j], t % 4) * s;
    }
  }
  const size_t at = ((size_t)r * Hkv + h) * D + d;
  if (out_k) q8_store4(out_k + at, k);
  if (out_v) q8_store4(out_v + at, v);
}

// Column sums of [m, L] in fixed point.  A workgroup takes 64 columns, its four waves every fourth of its rows.  Where several
// workgroups share columns they add with integer atomics: any order gives the same sum.
// What bounds it: launching and one or two latencies; 130 x 20001 5.0 us (10 MB).
__global__ __launch_bounds__(256) void q8_weigh_kernel(const float* avg, int m, int L, int rows_per_wg, unsigned long long* weight) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = blockIdx.x * 64 + lane;
  const int r0 = blockIdx.y * rows_per_wg, r1 = min(m, r0 + rows_per_wg);
  __shared__ unsigned long long part[3][64];
  unsigned long long sum = 0;
  if (j < L) {
#pragma unroll 8
    for (int r = r0 + wave; r < r1; r += 4) {
      const float c = fminf(fmaxf(avg[(size_t)r * L + j], 0.f), 1.f);
      sum += c >= 1.f ? 1ull << 32 : (unsigned long long)(uint32_t)(c * 4294967296.f);
    }
  }
  if (wave) part[wave - 1][lane] = sum;
  __syncthreads();
  if (wave || j >= L) return;
  sum += part[0][lane] + part[1][lane] + part[2][lane];
  if (gridDim.y == 1) weight[j] += sum;
  else if (sum) atomicAdd(&weight[j], sum);
}

// ---- the rows to keep: one workgroup of 16 waves
constexpr int kKeepWaves = 16, kKeepThreads = 64 * kKeepWaves;

// Wave w takes a run of positions, lane by lane; in registers where that is at most PER rounds of it (PER = 0: read again for each pass).
// The protected rows fill up first: if they are n_keep or more the choice is among them, else all of them stay and it is among the others.
// The chosen class's n-th largest weight is found digit by digit (11 bits, from its highest bit on), with a histogram in LDS and an early
// end when a digit's rows all stay.  Then each wave numbers its kept positions behind those of the waves before.
// What bounds it: a chain of barriers and LDS atomics per digit in one compute unit, and its instructions where there are many rows; 767 rows
// 6.3 us, 20001 16.4 (with equal keys told apart in every pass over them, not only where a part of them stays, 0.5 and 2.6 us more).
template <int PER, bool PROTECT>
__global__ __launch_bounds__(kKeepThreads) void q8_keep_kernel(const int64_t* weight, const uint8_t* protect, int L, int n_keep,
                                                              int32_t* kept, int64_t* kept_weight) {
  constexpr unsigned long long kTop = 1ull << 63;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rounds = ((L + kKeepWaves - 1) / kKeepWaves + 63) / 64, first = wave * rounds * 64 + lane;
  __shared__ uint32_t hist[2][2048], wave_sum[kKeepWaves], wave_bits[kKeepWaves], wave_up[kKeepWaves], wave_eq[kKeepWaves];
  __shared__ uint32_t found_bin, found_above, found_in;
  unsigned long long reg[PER ? PER : 1];                // weight, top bit: protected
  // (through buffers that end with the arrays, which answer 0 past them: loads under a condition would come one after the other.  The round
  // is part of the vector offset, which is compared with the buffer's end; the compiler's documentation leaves a scalar offset out of that)
  const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int64_t*>(weight), 0, L * 8, 0x00020000);
  const __amdgpu_buffer_rsrc_t p_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(protect), 0, PROTECT ? L : 0, 0x00020000);
  auto load = [&](int j) __attribute__((always_inline)) -> unsigned long long {
    const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(w_rsrc, (first + 64 * j) * 8, 0, 0);
    uint32_t hi = (int)w[1] < 0 ? 0u : w[1], lo = (int)w[1] < 0 ? 0u : w[0];
    if (PROTECT && __builtin_amdgcn_raw_buffer_load_b8(p_rsrc, first + 64 * j, 0, 0) != 0) hi |= 1u << 31;
    return (unsigned long long)hi << 32 | lo;
  };
  if constexpr (PER > 0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) reg[j] = load(j);
  }
  // f(key, whether there is one, round).  (`left` is opaque to the compiler in each pass: it would keep 20 comparisons' results for all of
  // them, and spill.)
  auto each = [&](auto f) __attribute__((always_inline)) {
    int left = L - first;
    asm volatile("" : "+v"(left));
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j < rounds) f(reg[j], 64 * j < left, j);
    } else {
      for (int j = 0; j < rounds; ++j) f(load(j), 64 * j < left, j);
    }
  };
  for (int b = tid; b < 2048; b += kKeepThreads) hist[0][b] = 0;
  // how many are protected, and how many bits each class's weights have
  uint32_t n_prot = 0;
  unsigned long long any[2] = {0, 0};
  each([&](unsigned long long k, bool valid, int) {
    k = valid ? k : 0ull;
    const unsigned long long p = PROTECT ? (unsigned long long)((long long)k >> 63) : 0ull;
    any[0] |= k & ~p;
    if (PROTECT) {
      any[1] |= k & p;
      n_prot += (uint32_t)(k >> 63);
    }
  });
  any[1] &= ~kTop;
  const uint32_t bits[2] = {(uint32_t)(any[0] ? 64 - __clzll((long long)any[0]) : 0), (uint32_t)(any[1] ? 64 - __clzll((long long)any[1]) : 0)};
  uint32_t both = bits[0] | bits[1] << 16;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t x = __shfl_xor(both, o, 64);
    both = max(both & 0xffffu, x & 0xffffu) | max(both & 0xffff0000u, x & 0xffff0000u);
    if (PROTECT) n_prot += __shfl_xor(n_prot, o, 64);
  }
  if (lane == 0) { wave_sum[wave] = n_prot; wave_bits[wave] = both; }
  __syncthreads();
  n_prot = both = 0;
#pragma unroll
  for (int w = 0; w < kKeepWaves; ++w) {
    const uint32_t x = wave_bits[w];
    n_prot += wave_sum[w];
    both = max(both & 0xffffu, x & 0xffffu) | max(both & 0xffff0000u, x & 0xffff0000u);
  }
  const bool among_protected = n_prot >= (uint32_t)n_keep;
  const unsigned long long cls = among_protected ? kTop : 0ull;                        // n_keep > 0
  uint32_t need = among_protected ? (uint32_t)n_keep : (uint32_t)n_keep - n_prot;      // of the class `cls`
  const uint32_t size = among_protected ? n_prot : (uint32_t)L - n_prot;
  // keys of the class above `thr` stay, of those equal to it under the mask of the digits looked at the first `need`: all of them, or, where
  // the last digit has been looked at, of equal keys the first
  unsigned long long thr = cls, mask = kTop;
  bool some = false;
  if (need < size) {
    some = true;
    int hi = among_protected ? both >> 16 : both & 0xffffu;     // bits hi .. 62 are 0 throughout
    mask = ~0ull << hi;
    for (int pass = 0; hi > 0; ++pass) {
      const int lo = max(0, hi - 11);
      const uint32_t bins = 1u << (hi - lo);
      uint32_t* h = hist[pass & 1];
      each([&](unsigned long long k, bool valid, int) { if (valid && (k & mask) == thr) atomicAdd(&h[(uint32_t)(k >> lo) & (bins - 1)], 1u); });
      for (int b = tid; b < 2048; b += kKeepThreads) hist[(pass & 1) ^ 1][b] = 0;
      __syncthreads();
      // thread t holds bins 2047 - 2t and below: prefix sums run from the largest digit down
      const uint32_t a = h[2047 - 2 * tid], c = h[2046 - 2 * tid];
      uint32_t s = a + c;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = __shfl_up(s, o, 64);
        if (lane >= o) s += t;
      }
      if (lane == 63) wave_sum[wave] = s;
      __syncthreads();
      uint32_t before = s - a - c;
#pragma unroll
      for (int w = 0; w < kKeepWaves; ++w) before += w < wave ? wave_sum[w] : 0u;
      if (before < need && before + a >= need) { found_bin = 2047 - 2 * tid; found_above = before; found_in = a; }
      else if (before + a < need && before + a + c >= need) { found_bin = 2046 - 2 * tid; found_above = before + a; found_in = c; }
      __syncthreads();
      need -= found_above;
      thr |= (unsigned long long)found_bin << lo;
      mask = ~0ull << lo;
      hi = lo;
      some = need != found_in;
      if (!some) break;
    }
  }
  uint32_t n_up = 0, n_eq = 0;
  if (some) {
    each([&](unsigned long long k, bool valid, int) {
      n_up += __popcll(__ballot(valid && k > thr));
      n_eq += __popcll(__ballot(valid && k == thr));
    });
  } else {
    each([&](unsigned long long k, bool valid, int) { n_up += __popcll(__ballot(valid && k >= thr)); });
  }
  if (lane == 0) { wave_up[wave] = n_up; wave_eq[wave] = n_eq; }
  __syncthreads();
  uint32_t up = 0, eq = 0;
#pragma unroll
  for (int w = 0; w < kKeepWaves; ++w) {
    up += w < wave ? wave_up[w] : 0u;
    eq += w < wave ? wave_eq[w] : 0u;
  }
  auto put = [&](uint32_t at, int j, unsigned long long key) __attribute__((always_inline)) {
    kept[at] = first + 64 * j;
    if (kept_weight) kept_weight[at] = (int64_t)(key & ~kTop);
  };
  auto below = [](uint64_t b) { return (uint32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0u)); };
  if (some) {
    each([&](unsigned long long key, bool valid, int j) {
      const bool is_up = valid && key > thr, is_eq = valid && key == thr;
      const uint64_t u = __ballot(is_up), e = __ballot(is_eq);
      const uint32_t eq_at = eq + below(e);
      if (is_up || (is_eq && eq_at < need)) put(up + below(u) + min(eq_at, need), j, key);
      up += __popcll(u);
      eq += __popcll(e);
    });
  } else {
    each([&](unsigned long long key, bool valid, int j) {
      const bool stays = valid && key >= thr;
      const uint64_t u = __ballot(stays);
      if (stays) put(up + below(u), j, key);
      up += __popcll(u);
    });
  }
}

// Row i of dst is row kept[i] of src.  A workgroup per (block of dst, kv head, K or V): 16 KB read (V: more, its pieces hold four rows
// of which some go), 8 KB written.  What bounds it: the chain kept -> scales -> rows; 500 rows of 32 heads of 128 7.6 us, 9999 of 4 heads 10.3.
template <int D>
__global__ __launch_bounds__(256) void q8_compact_kernel(Q8CachePtr src, const int32_t* kept, int n, Q8CachePtr dst, int Hkv) {
  using P = Pieces<D>;
  const int b = blockIdx.x, h = blockIdx.y >> 1, is_v = blockIdx.y & 1, tid = threadIdx.x;
  __shared__ int from[kQ8Rows];
  __shared__ float scale_of[kQ8Rows];
  const uint8_t* codes = is_v ? src.v : src.k;
  if (tid < kQ8Rows) {
    const int i = b * kQ8Rows + tid, pos = i < n ? kept[i] : -1;
    from[tid] = pos;
    scale_of[tid] = pos >= 0 ? (is_v ? src.vs : src.ks)[(size_t)(pos / kQ8Rows) * Hkv + h] : 0.f;
  }
  __syncthreads();
  const float s = wave_max(scale_of[tid & 63]), inv = q8_inverse(s);
  // (places past the last are read as the first row and set to code 0)
  uint8_t* out = (is_v ? dst.v : dst.k) + ((size_t)b * Hkv + h) * kQ8Rows * D;
#pragma unroll
  for (int i = 0; i < P::kPerThread; ++i) {
    const int p = tid + 256 * i;
    u32x4 r;
    if (is_v) {
      u32x4 w[4];
      float old[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int pos = max(from[P::v_row(p) + j], 0);
        old[j] = scale_of[P::v_row(p) + j];
        w[j] = ld16(codes + ((size_t)(pos / kQ8Rows) * Hkv + h) * kQ8Rows * D + pos % kQ8Rows / 4 * 4 * D + P::v_dim(p) * 4);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = P::v_row(p) + j;
        // the row's bytes of its four words, as one word
        const uint32_t sel = 0x0c0c0000u | (from[t] & 3) | (4 + (from[t] & 3)) << 8;
        uint32_t x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[j][3], w[j][2], sel), __builtin_amdgcn_perm(w[j][1], w[j][0], sel), 0x05040100u);
        if (old[j] != s) x = q8_reword(x, old[j], s, inv, old[j] * inv);
        if (from[t] < 0) x = 0x80808080u;
        w[j][0] = x;
      }
      // four rows of four dimensions -> four dimensions of four rows
      const uint32_t lo0 = __builtin_amdgcn_perm(w[1][0], w[0][0], 0x05010400u), lo1 = __builtin_amdgcn_perm(w[1][0], w[0][0], 0x07030602u);
      const uint32_t hi0 = __builtin_amdgcn_perm(w[3][0], w[2][0], 0x05010400u), hi1 = __builtin_amdgcn_perm(w[3][0], w[2][0], 0x07030602u);
      r[0] = __builtin_amdgcn_perm(hi0, lo0, 0x05040100u);
      r[1] = __builtin_amdgcn_perm(hi0, lo0, 0x07060302u);
      r[2] = __builtin_amdgcn_perm(hi1, lo1, 0x05040100u);
      r[3] = __builtin_amdgcn_perm(hi1, lo1, 0x07060302u);
      *reinterpret_cast<u32x4*>(out + P::v_at(p)) = r;
    } else {
      const int t = P::k_row(p), pos = max(from[t], 0);
      r = ld16(codes + ((size_t)(pos / kQ8Rows) * Hkv + h) * kQ8Rows * D + P::k_dim(p) * kQ8Rows + pos % kQ8Rows * 16);
      const float old = scale_of[t], ratio = old * inv;
      if (old != s)
#pragma unroll
        for (int d = 0; d < 4; ++d) r[d] = q8_reword(r[d], old, s, inv, ratio);
      if (from[t] < 0) r = u32x4{0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
      *reinterpret_cast<u32x4*>(out + P::k_at(p)) = r;
    }
  }
  if (tid == 0) (is_v ? dst.vs : dst.ks)[(size_t)b * Hkv + h] = s;
}

template <typename T>
hipError_t update_t(const Q8Shape& s, const UpdateArgs& a, dim3 grid, hipStream_t st) {
  if (s.D == 128) q8_update_kernel<T, 128><<<grid, 256, 0, st>>>(a, s.Hkv);
  else q8_update_kernel<T, 64><<<grid, 256, 0, st>>>(a, s.Hkv);
  return hipGetLastError();
}

template <typename T>
hipError_t read_t(const Q8Shape& s, const Q8CachePtr& c, int L, const int32_t* idx, int n, void* k, void* v, hipStream_t st) {
  const int rows = 1024 / s.D;
  const dim3 grid((n + rows - 1) / rows, s.Hkv);
  if (s.D == 128) q8_read_kernel<T, 128><<<grid, 256, 0, st>>>(c, L, idx, n, s.Hkv, (T*)k, (T*)v);
  else q8_read_kernel<T, 64><<<grid, 256, 0, st>>>(c, L, idx, n, s.Hkv, (T*)k, (T*)v);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_update(const Q8Shape& s, const Q8Update* calls, int n, hipStream_t st) {
  for (int c0 = 0; c0 < n; c0 += kQ8Launch) {
    UpdateArgs a{};
    const int nc = std::min(kQ8Launch, n - c0);
    int slots = 0;
    for (int i = 0; i < nc; ++i) {
      a.c[i] = calls[c0 + i];
      const int nb = q8_blocks(a.c[i].L), first = (a.c[i].L - a.c[i].m) / kQ8Rows;
      slots = std::max(slots, a.c[i].idx ? std::min(a.c[i].m, nb) : nb - first);
    }
    const dim3 grid(slots, 2 * s.Hkv, nc);
    const hipError_t e = s.dtype == kBF16 ? update_t<bf16>(s, a, grid, st) : update_t<float>(s, a, grid, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_q8_read(const Q8Shape& s, const Q8CachePtr& c, int L, const int32_t* idx, int n, void* k, void* v, hipStream_t st) {
  return s.dtype == kBF16 ? read_t<bf16>(s, c, L, idx, n, k, v, st) : read_t<float>(s, c, L, idx, n, k, v, st);
}

hipError_t launch_q8_weigh(const float* avg, int m, int L, int64_t* weight, hipStream_t st) {
  const int cols = (L + 63) / 64;
  const int parts = std::max(1, std::min((m + 15) / 16, 1024 / cols));
  const int per = (m + parts - 1) / parts;
  q8_weigh_kernel<<<dim3(cols, (m + per - 1) / per), 256, 0, st>>>(avg, m, L, per, (unsigned long long*)weight);
  return hipGetLastError();
}

hipError_t launch_q8_keep(const int64_t* weight, const uint8_t* protect, int L, int n_keep, int32_t* kept, int64_t* kept_weight,
                          hipStream_t st) {
  // Rounds of a wave.  Rounds that are not there cost nearly what others do, and keys that are read again their way from the L2.  A call that keeps
  // 64 rows of one head (choice and compaction, in a captured loop), us, with protected rows:
  //   rows              767  2000  4096  4097  5000  6000  8000  10000  12000  16000  20001  20480
  //   4 in registers    7.4   7.6   8.2
  //   20 in registers  11.1  11.3  11.8  12.0  12.0  12.3  12.8   15.2   13.4   14.5   17.8   15.4
  //   read again        7.5   8.5  10.0  10.7  10.9  11.7  13.2   17.7   16.3   19.0   26.7   22.2
  const int per = ((L + kKeepWaves - 1) / kKeepWaves + 63) / 64;
  auto go = [&](auto prot) {
    constexpr bool P = decltype(prot)::value;
    if (per <= 4) q8_keep_kernel<4, P><<<1, kKeepThreads, 0, st>>>(weight, protect, L, n_keep, kept, kept_weight);
    else if (per > 6 && per <= 20) q8_keep_kernel<20, P><<<1, kKeepThreads, 0, st>>>(weight, protect, L, n_keep, kept, kept_weight);
    else q8_keep_kernel<0, P><<<1, kKeepThreads, 0, st>>>(weight, protect, L, n_keep, kept, kept_weight);
    return hipGetLastError();
  };
  return protect ? go(std::true_type{}) : go(std::false_type{});
}

hipError_t launch_q8_compact(const Q8Shape& s, const Q8CachePtr& src, const int32_t* kept, int n, const Q8CachePtr& dst,
                             hipStream_t st) {
  const dim3 grid(q8_blocks(n), 2 * s.Hkv);
  if (s.D == 128) q8_compact_kernel<128><<<grid, 256, 0, st>>>(src, kept, n, dst, s.Hkv);
  else q8_compact_kernel<64><<<grid, 256, 0, st>>>(src, kept, n, dst, s.Hkv);
  return hipGetLastError();
}

}  // namespace d2c
