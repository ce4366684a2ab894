// Products in 8-bit integers: out[m, N] = (sum_k qa[m, k] qw[n, k]) sa[m] sw[n], exact sums in 32 bits.
//
// Both operands lie in the order in which the matrix cores take them (v_mfma_i32_16x16x64_i8): tiles of 16 rows x 64 of the
// contraction, 1 KB each, lane l's 16 bytes (row l % 16, contraction 16 (l / 16) ..) at 16 l; rows and contraction are padded with
// zeros to whole tiles.  Weights are brought into that order once, activations in a launch of their own in front of each product (both
// q8_rows_kernel), with a scale per row; a few short rows are rounded inside the product's launch.
#include <algorithm>

#include "q8.h"

namespace d2c {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Rows quantised by their largest magnitude; a row that holds a NaN or an infinity gets the scale NaN and codes 0.  What pads
// the last tile is not written, or holds the last row again: it gives outputs that nothing stores.
//
// A workgroup takes a row, or a part of its columns (blockIdx.y) while there are few rows, 16 columns per thread at a time: one lane's piece
// of a tile.  It looks at the whole row for its largest magnitude -- integer maxima of the bits without sign: infinities and NaN are the
// largest -- and rounds its part from registers.  What bounds it: one chain of load, maximum, barrier and store; 37 x 18944 5 us, 1536 x
// 4096 10 us (4 waves a row; 16 waves 17).  Sixteen rows per workgroup with lanes as in a tile, so that codes leave a kilobyte
// at a time, took longer (22 and 18 us): their loads are 128-byte pieces of 16 rows.
//
// Rounding: the sum with 1.5 * 2^23 leaves the whole number nearest to x / s (or its neighbour, next to a border) in its low byte, and the
// remainder x - n s, which has no rounding (see q8_code), says if all 16 are the nearest: only where a remainder is half a step or more
// are they done with care.
template <typename T> struct Raw16;
template <> struct Raw16<bf16> {
  u32x4 w[2];
  __device__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = w[i / 4][i % 4] & 0x7fff7fffu;
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, x)));
    }
    return max(m << 16, m & 0xffff0000u);
  }
  __device__ float at(int i) const {
    const uint32_t x = w[i / 8][i / 2 % 4];
    return __builtin_bit_cast(float, i & 1 ? x & 0xffff0000u : x << 16);
  }
};
template <> struct Raw16<float> {
  u32x4 w[4];
  __device__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, w[i / 4][i % 4] & 0x7fffffffu);
    return m;
  }
  __device__ float at(int i) const {
    const uint32_t x = w[i / 4][i % 4];
    return __builtin_bit_cast(float, x);
  }
};
// (read from a place inside where there is nothing, and set to 0 afterwards: loads under a condition would come one after the other)
template <typename T>
__device__ __forceinline__ Raw16<T> load16(const T* row, int k, int K) {
  constexpr int kEach = 16 / sizeof(T), kN = sizeof(Raw16<T>) / 16;         // K is a multiple of 16 bytes
  Raw16<T> v;
#pragma unroll
  for (int i = 0; i < kN; ++i) v.w[i] = ld16(row + min(k + i * kEach, K - kEach));
  return v;
}
template <typename T>
__device__ __forceinline__ void zero_past(Raw16<T>& v, int k, int K) {
  constexpr int kEach = 16 / sizeof(T), kN = sizeof(Raw16<T>) / 16;
#pragma unroll
  for (int i = 0; i < kN; ++i)
    if (k + i * kEach >= K) v.w[i] = u32x4{0, 0, 0, 0};
}
template <typename T>
__device__ __forceinline__ u32x4 round16(const Raw16<T>& v, float s, float inv) {
  constexpr float kMagic = 12582912.f;
  const float border = 0.5f * s;
  float worst = 0.f;
  u32x4 c;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = v.at(4 * q + j), n = fmaf(x, inv, kMagic);
      worst = fmaxf(worst, fabsf(fmaf(-(n - kMagic), s, x)));
      b[j] = __builtin_bit_cast(uint32_t, n);
    }
    c[q] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
  }
  if (worst >= border) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      c[q] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c[q] |= (uint32_t)(uint8_t)q8_code(v.at(4 * q + j), s, inv) << (8 * j);
    }
  }
  return c;
}
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}
// the scale that a row's largest bits give, the row's scale as it is stored, and the codes of a piece
struct RowScale {
  float s, inv;
  bool bad;
  __device__ explicit RowScale(uint32_t bits) : bad(bits >= 0x7f800000u) {
    s = bad ? 0.f : q8_scale(__builtin_bit_cast(float, bits));
    inv = q8_inverse(s);
  }
  __device__ float stored() const { return bad ? __builtin_nanf("") : s; }
  template <typename T> __device__ void put(int8_t* to, const Raw16<T>& w) const {
    u32x4 c = {0, 0, 0, 0};
    if (s > 0.f) c = round16(w, s, inv);
    *reinterpret_cast<u32x4*>(to) = c;
  }
};

template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void q8_rows_kernel(const T* x, int K, int kc, int per_part, int8_t* codes, float* scale) {
  const int r = blockIdx.x, tid = threadIdx.x;
  const T* row = x + (size_t)r * K;
  const int p0 = blockIdx.y * per_part, p1 = min(4 * kc, p0 + per_part);      // pieces of 16 columns
  __shared__ uint32_t red[WAVES];
  Raw16<T> v = load16(row, 16 * (p0 + tid), K);
  zero_past(v, 16 * (p0 + tid), K);
  uint32_t bits = v.largest();
  // what this part has not in registers (what load16 repeats at the end is the row's own)
  for (int p = tid; 16 * p < K; p += 64 * WAVES)
    if (p < p0 || p >= p0 + 64 * WAVES) bits = max(bits, load16(row, 16 * p, K).largest());
  bits = wave_max_bits(bits);
  if ((tid & 63) == 0) red[tid >> 6] = bits;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) bits = max(bits, red[w]);
  const RowScale s(bits);
  if (tid == 0 && p0 == 0) scale[r] = s.stored();
  int8_t* to = codes + (size_t)(r / 16) * kc * 1024 + r % 16 * 16;
  auto at = [&](int p) { return to + (size_t)(p / 4) * 1024 + p % 4 * 256; };
  if (p0 + tid < p1) s.put(at(p0 + tid), v);
  for (int p = p0 + tid + 64 * WAVES; p < p1; p += 64 * WAVES) {
    v = load16(row, 16 * p, K);
    zero_past(v, 16 * p, K);
    s.put(at(p), v);
  }
}

__device__ __forceinline__ i32x4 mfma_i8(const u32x4& a, const u32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Few rows: the weights stream past once.  A workgroup takes NT tiles of 16 outputs and up to MT tiles of 16 rows, its waves every
// WAVES-th step of 64 of the contraction, so that together they read consecutive kilobytes; the next UNROLL steps' weights are on their way
// while one step's activations come from the L2.  The waves' sums are whole numbers and are added up in LDS in any order.  With few
// outputs the contraction is split over workgroups too (blockIdx.y) and q8_sum_kernel adds the parts.
template <int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void q8_stream_kernel(const int8_t* a, const float* sa, const int8_t* w, const float* sw, int m,
                                                               int N, int kc, int ka, int k_per, float* out, int* part) {
  constexpr int U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m_tiles = (m + 15) / 16, n_tiles = (N + 15) / 16;
  const int nt0 = blockIdx.x * NT, k0 = blockIdx.y * k_per, k1 = min(kc, k0 + k_per);
  __shared__ int sums[NT][MT][256];
  for (int i = threadIdx.x; i < NT * MT * 256; i += 64 * WAVES) (&sums[0][0][0])[i] = 0;
  __syncthreads();
  const int8_t *wp[NT], *ap[MT];
#pragma unroll
  for (int n = 0; n < NT; ++n) wp[n] = w + (size_t)min(nt0 + n, n_tiles - 1) * kc * 1024 + lane * 16;
#pragma unroll
  for (int t = 0; t < MT; ++t) ap[t] = a + (size_t)min(t, m_tiles - 1) * ka * 1024 + lane * 16;
  i32x4 acc[NT][MT] = {};
  u32x4 wf[U][NT];
  auto fetch = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) wf[u][n] = ld16(wp[n] + (size_t)min(k + u * WAVES, kc - 1) * 1024);
  };
  int k = k0 + wave;
  fetch(k);
  for (; k + (U - 1) * WAVES < k1; k += U * WAVES) {
    u32x4 now[U][NT], af[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) now[u][n] = wf[u][n];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t) af[u][t] = ld16(ap[t] + (size_t)(k + u * WAVES) * 1024);
    fetch(k + U * WAVES);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][t] = mfma_i8(now[u][n], af[u][t], acc[n][t]);
  }
#pragma unroll
  for (int u = 0; u < U - 1; ++u) {
    const int ku = k + u * WAVES;
    if (ku < k1) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const u32x4 af = ld16(ap[t] + (size_t)ku * 1024);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][t] = mfma_i8(wf[u][n], af, acc[n][t]);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) atomicAdd(&sums[n][t][j * 64 + lane], acc[n][t][j]);
  __syncthreads();
  // a piece: four outputs of a row
  for (int p = threadIdx.x; p < NT * MT * 64; p += 64 * WAVES) {
    const int l = p & 63, t = p / 64 % MT, n = p / 64 / MT;
    const int row = t * 16 + l % 16, col = (nt0 + n) * 16 + l / 16 * 4;
    if (row >= m || col >= N) continue;
    i32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = sums[n][t][j * 64 + l];
    if (part) {
      int* to = part + ((size_t)blockIdx.y * m + row) * N + col;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < N) to[j] = v[j];
    } else {
      const float s = sa[row];
      float* to = out + (size_t)row * N + col;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < N) to[j] = (float)v[j] * s * sw[col + j];
    }
  }
}

// Up to 16 rows and a short contraction (kc <= 32): one launch.  Every workgroup rounds all the rows into LDS by itself, a wave a row, while
// its weights -- a tile of 16 outputs, two steps of the contraction per wave at most -- are on their way.
// What bounds it: launching, and one chain of load, maximum, code, barrier, product, barrier (times in launch_q8_linear).
template <typename T>
__global__ __launch_bounds__(1024) void q8_small_kernel(const T* x, const int8_t* w, const float* sw, int m, int N, int K, int kc, float* out) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  __shared__ __attribute__((aligned(16))) int8_t codes[32 * 1024];      // [step][1 KB]
  __shared__ int sums[256];
  __shared__ float scale[16];
  const int8_t* wp = w + (size_t)blockIdx.x * kc * 1024 + lane * 16;
  u32x4 wf[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) wf[u] = ld16(wp + (size_t)min(wave + 16 * u, kc - 1) * 1024);
  if (threadIdx.x < 256) sums[threadIdx.x] = 0;
  const T* row = x + (size_t)min(wave, m - 1) * K;                      // past the last row that one again, not stored
  Raw16<T> v[2];
  uint32_t bits = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) v[u] = load16(row, 16 * (lane + 64 * u), K);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    zero_past(v[u], 16 * (lane + 64 * u), K);
    bits = max(bits, v[u].largest());
  }
  const RowScale s(wave_max_bits(bits));
  if (lane == 0) scale[wave] = s.stored();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int p = lane + 64 * u;
    if (p < 4 * kc) s.put(codes + p / 4 * 1024 + p % 4 * 256 + wave * 16, v[u]);
  }
  __syncthreads();
  i32x4 acc = {};
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = wave + 16 * u;
    if (k < kc) acc = mfma_i8(wf[u], *reinterpret_cast<const u32x4*>(codes + k * 1024 + lane * 16), acc);
  }
  if (wave < kc)
#pragma unroll
    for (int j = 0; j < 4; ++j) atomicAdd(&sums[j * 64 + lane], acc[j]);
  __syncthreads();
  const int r = lane % 16, col = blockIdx.x * 16 + lane / 16 * 4;
  if (wave || r >= m) return;
  float* to = out + (size_t)r * N + col;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < N) to[j] = (float)sums[j * 64 + lane] * scale[r] * sw[col + j];
}

// out = the parts' sums, scaled.  A workgroup per (row, 256 outputs): with one index over all outputs, and its division by N, a call of
// 37 x 3584 x 18944 (eight parts) took 22.5 us, this way 21.2.  What bounds it: launching and one latency.
__global__ __launch_bounds__(256) void q8_sum_kernel(const int* part, int splits, const float* sa, const float* sw, int m, int N, float* out) {
  const int row = blockIdx.x, col = blockIdx.y * 256 + threadIdx.x;
  if (col >= N) return;
  const size_t total = (size_t)m * N;
  const int* from = part + (size_t)row * N + col;
  const float s = sa[row], n = sw[col];
  int v = 0;
#pragma unroll 4
  for (int i = 0; i < splits; ++i) v += from[i * total];
  out[(size_t)row * N + col] = (float)v * s * n;
}

// Many rows: matrix-core bound.  A workgroup of 8 waves computes 16 MT rows x 128 NT outputs, each wave all the rows and 16 NT outputs of
// its own, so that a weight is asked of the L1 once (two waves over the rows and four over the outputs: 1536 x 24576 x 4096 191 us,
// this way 177).  Activations, which all waves read, go straight into LDS in chunks of four steps of the contraction; weights come into
// registers from the order they lie in and are refilled as soon as a step is done.  LDS reads run three groups of NT matrix-core instructions
// ahead of their use.  Each XCD takes a run of tiles in an order in which neighbours share activations and weights in its L2.  Splits of the
// contraction write their sums to `part`.
// What bounds it: the matrix cores, busy 62 % of the time that waves are there (1536 x 24576 x 4096: 146-162 us, 1.9-2.1 POP/s), and the barrier of each chunk,
// with one workgroup per compute unit: waves wait 34 % of their time.  Two chunks on their way instead of one gave nothing.
constexpr int kStepsPerChunk = 4;
template <int MT, int NT>
__global__ __launch_bounds__(512, 1) void q8_tile_kernel(const int8_t* a, const float* sa, const int8_t* w, const float* sw, int m, int N,
                                                         int kc, int ka, int chunks_per, int row_groups, int col_groups, int splits,
                                                         float* out, int* part) {
  constexpr int kBuf = MT * kStepsPerChunk * 1024, kBlocks = MT * kStepsPerChunk, kStage = (kBlocks + 7) / 8, kCols = 4;
  constexpr int kPitch = 128 * NT + 4, kOut = 16 * kPitch * 4;       // outputs on their way: 16 rows; the pitch takes them to other banks
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * kBuf > 2 * kOut ? 2 * kBuf : 2 * kOut];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m_tiles = (m + 15) / 16, n_tiles = (N + 15) / 16;
  // id % 8 is the XCD; its run of tiles goes down the row groups over kCols column groups at a time
  const int all_cols = col_groups * splits, total = row_groups * all_cols, per_xcd = (total + 7) / 8;
  const int id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || id >= total) return;            // whole workgroups
  const int band = id / (row_groups * kCols), width = min(kCols, all_cols - band * kCols), in = id - band * row_groups * kCols;
  const int rg = in / width, tile = band * kCols + in % width;
  const int split = tile / col_groups, cg = tile % col_groups;
  const int mt0 = rg * MT, nt0 = (cg * 8 + wave) * NT;
  const int c0 = split * chunks_per, n_chunks = min(ka / kStepsPerChunk - c0, chunks_per);

  const int8_t* wp[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) wp[n] = w + (size_t)min(nt0 + n, n_tiles - 1) * kc * 1024 + lane * 16;
  // staging: block wave + 8 i is step (that) % 4 of row tile (that) / 4 (tiles past the last row repeat it)
  unsigned aoff[kStage];
#pragma unroll
  for (int i = 0; i < kStage; ++i) {
    const int blk = wave + 8 * i;
    aoff[i] = ((unsigned)min(blk / kStepsPerChunk, m_tiles - 1 - mt0) * ka + blk % kStepsPerChunk) * 1024u + lane * 16;
  }
  // (the workgroup's rows, 8 MB at most: offsets have 32 bits)
  const __amdgpu_buffer_rsrc_t arsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a) + (size_t)mt0 * ka * 1024, 0,
                                                                         min(MT, m_tiles - mt0) * ka * 1024, 0x00020000);
  auto stage = [&](int buf, int chunk) {
#pragma unroll
    for (int i = 0; i < kStage; ++i)
      if (kBlocks % 8 == 0 || wave + 8 * i < kBlocks)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(arsrc, (__attribute__((address_space(3))) void*)(lds + buf * kBuf + (wave + 8 * i) * 1024), 16,
                                               (int)aoff[i], chunk * kStepsPerChunk * 1024, 0, 0);
  };
  u32x4 b[NT][kStepsPerChunk];
  auto load_b = [&](int chunk, int step) __attribute__((always_inline)) {   // steps past the weights' own meet zeros
    const size_t off = (size_t)min(chunk * kStepsPerChunk + step, kc - 1) * 1024;
#pragma unroll
    for (int n = 0; n < NT; ++n) b[n][step] = ld16(wp[n] + off);
  };
  i32x4 acc[MT][NT] = {};
  const int last = c0 + n_chunks - 1;
  stage(0, c0);
#pragma unroll
  for (int s = 0; s < kStepsPerChunk; ++s) load_b(c0, s);
  __builtin_amdgcn_sched_barrier(0);
  // a chunk is in LDS once the weights that were requested behind its staging are all that is missing
  constexpr int kBehind = kStepsPerChunk * NT;
  auto wait = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt((kBehind & 15) | ((kBehind >> 4) << 14) | 0x70 | 0xf00);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  wait();
  constexpr int NI = kStepsPerChunk * MT;
  for (int c = 0; c < n_chunks; ++c) {
    const int next = min(c0 + c + 1, last);                // behind the last chunk that one again, not used
    stage((c & 1) ^ 1, next);
    __builtin_amdgcn_sched_barrier(0);
    const unsigned char* abuf = lds + (c & 1) * kBuf + lane * 16;
    auto read_a = [&](int i) { return *reinterpret_cast<const u32x4*>(abuf + (i % MT * kStepsPerChunk + i / MT) * 1024); };
    u32x4 af[4];
    af[0] = read_a(0);
    af[1] = read_a(1);
    af[2] = read_a(2);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[i % MT][n] = mfma_i8(b[n][i / MT], af[i % 4], acc[i % MT][n]);
      if (i + 3 < NI) af[(i + 3) % 4] = read_a(i + 3);
      if (i % MT == MT - 1) load_b(next, i / MT);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, NT, 0);
      if (i + 3 < NI) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (i % MT == MT - 1) __builtin_amdgcn_sched_group_barrier(0x020, NT, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    wait();
  }
  __builtin_amdgcn_s_waitcnt(0x70 | 0xf00);                 // no staging may write LDS any more
  __syncthreads();
  // Outputs leave through LDS, 16 rows at a time, in whole rows of the workgroup's columns: from the accumulators they would leave in
  // pieces of 64 bytes (1536 x 24576 x 4096 178 us, this way 157)
  float sn[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = (nt0 + n) * 16 + lane / 16 * 4 + j;
      sn[n][j] = col < N ? sw[col] : 0.f;
    }
  const int row_base = mt0 * 16, col_base = cg * 8 * NT * 16;
  int* to = (part ? part + (size_t)split * m * N : (int*)out) + (size_t)row_base * N + col_base;
  const bool whole = N % 4 == 0 && ((uintptr_t)to & 15) == 0;              // four outputs of a row are 16 aligned bytes
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    int* o = (int*)(lds + (t & 1) * kOut);
    const float r = sa[min(row_base + t * 16 + lane % 16, m - 1)];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      i32x4 y = acc[t][n];
      if (!part) {
        f32x4 f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = (float)y[j] * r * sn[n][j];
        y = __builtin_bit_cast(i32x4, f);
      }
      *reinterpret_cast<i32x4*>(o + lane % 16 * kPitch + (wave * NT + n) * 16 + lane / 16 * 4) = y;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int p = threadIdx.x + 512 * i, row = p / (32 * NT), col = p % (32 * NT) * 4;
      if (row_base + t * 16 + row >= m || col_base + col >= N) continue;
      const i32x4 y = *reinterpret_cast<const i32x4*>(o + row * kPitch + col);
      int* at = to + (size_t)(t * 16 + row) * N + col;
      if (whole) {
        *reinterpret_cast<i32x4*>(at) = y;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col_base + col + j < N) at[j] = y[j];
      }
    }
  }
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr size_t kPartBytes = (size_t)32 << 20;       // room for the parts of split contractions
constexpr int kStreamRows = 32;

// kc: steps of the contraction in the weights' layout, ka: in the activations' (whole chunks)
struct Operands { const int8_t* a; const float* sa; const int8_t* w; const float* sw; int m, N, kc, ka; float* out; int* part; };

hipError_t sum_parts(const Operands& o, int splits, hipStream_t st) {
  q8_sum_kernel<<<dim3(o.m, (o.N + 255) / 256), 256, 0, st>>>(o.part, splits, o.sa, o.sw, o.m, o.N, o.out);
  return hipGetLastError();
}
// splits: a workgroup for each compute unit, while each wave has two steps and more and the parts have room
int plan_stream(int m, int N, int kc, int nt, int waves) {
  const int groups = ((N + 15) / 16 + nt - 1) / nt;
  int splits = 1;
  while (groups * splits * 2 <= 256 && kc / (2 * splits) >= 2 * waves && (size_t)2 * splits * m * N * 4 <= kPartBytes) splits *= 2;
  return splits;
}
template <int MT, int NT, int WAVES>
hipError_t stream(const Operands& o, int splits, hipStream_t st) {
  const int groups = ((o.N + 15) / 16 + NT - 1) / NT, per = (o.kc + splits - 1) / splits;
  q8_stream_kernel<MT, NT, WAVES><<<dim3(groups, splits), 64 * WAVES, 0, st>>>(o.a, o.sa, o.w, o.sw, o.m, o.N, o.kc, o.ka, per, o.out,
                                                                                splits > 1 ? o.part : nullptr);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || splits == 1 ? e : sum_parts(o, splits, st);
}
template <int MT, int NT>
hipError_t tile(const Operands& o, int splits, hipStream_t st) {
  const int rows = 16 * MT, cols = 128 * NT, rg = (o.m + rows - 1) / rows, cg = (o.N + cols - 1) / cols, chunks = o.ka / kStepsPerChunk;
  const int per = (chunks + splits - 1) / splits;
  const int per_xcd = (rg * cg * splits + 7) / 8;
  q8_tile_kernel<MT, NT><<<8 * per_xcd, 512, 0, st>>>(o.a, o.sa, o.w, o.sw, o.m, o.N, o.kc, o.ka, per, rg, cg, splits, o.out,
                                                      splits > 1 ? o.part : nullptr);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || splits == 1 ? e : sum_parts(o, splits, st);
}

// The tile kernel's shape and splits by an estimate of its time in us, fitted to 159 sizes (33-1536 rows, 64-37888 outputs, contractions of
// 64-18944; all shapes and splits measured on each).  A round of workgroups starts in `round`; a chunk takes a workgroup c0 + c1 MT NT +
// c2 NT, and as long as its bytes take from the L2 where all compute units pull; then its outputs' way to memory.  Splits cost a
// launch and the parts' way out and in.  What it picks is 1.0 % behind the best on average, 16 % at most; always taking MT = 8, NT = 2
// without splits is 50 % behind at 128 rows and more.
Q8LinearPlan plan_tile(int m, int N, int ka) {
  constexpr float round = 0.83f, c0 = 0.29f, c1 = 0.09f, c2 = 0.04f, l2 = 120.f, out = 0.55f, split_launch = 2.7f, split_bytes = 5.5e6f;
  static constexpr int8_t shapes[][2] = {{1, 1}, {2, 1}, {3, 1}, {4, 1}, {6, 1}, {8, 1}, {4, 2}, {6, 2}, {8, 2}, {8, 3}};
  static constexpr int8_t counts[] = {1, 2, 3, 4, 6, 8, 12};
  const int chunks = ka / kStepsPerChunk, m_tiles = (m + 15) / 16;
  Q8LinearPlan best{kQ8Tile, 8, 2, 8, 1};
  float best_cost = 1e30f;
  for (const auto& sh : shapes) {
    const int mt = sh[0], nt = sh[1];
    if (mt > 1 && mt / 2 >= m_tiles) continue;            // more than half of the rows idle
    const int groups = ((m_tiles + mt - 1) / mt) * ((N + 128 * nt - 1) / (128 * nt));
    if (mt < 4 && groups > 2048) continue;                // not measured
    for (int n : counts) {
      if (n > 1 && (n > chunks || (size_t)n * m * N * 4 > kPartBytes || groups * n > 1024)) break;
      const int per = (chunks + n - 1) / n, splits = (chunks + per - 1) / per, wgs = groups * splits;
      const float share = std::min(1.f, wgs / 256.f);
      const float chunk = std::max(c0 + c1 * mt * nt + c2 * nt, 4.f * (mt + 8 * nt) / l2 * share);
      float cost = (wgs + 255) / 256 * (round + per * chunk + out * mt * nt * share);
      if (splits > 1) cost += split_launch + 8.f * splits * m * N / split_bytes;
      if (cost < best_cost) { best_cost = cost; best = Q8LinearPlan{kQ8Tile, mt, nt, 8, splits}; }
    }
  }
  return best;
}
hipError_t run_tile(const Operands& o, const Q8LinearPlan& p, hipStream_t st) {
  if (p.nt == 3) return tile<8, 3>(o, p.splits, st);
  if (p.nt == 2) return p.mt == 4 ? tile<4, 2>(o, p.splits, st) : p.mt == 6 ? tile<6, 2>(o, p.splits, st) : tile<8, 2>(o, p.splits, st);
  switch (p.mt) {
    case 1: return tile<1, 1>(o, p.splits, st);
    case 2: return tile<2, 1>(o, p.splits, st);
    case 3: return tile<3, 1>(o, p.splits, st);
    case 4: return tile<4, 1>(o, p.splits, st);
    case 6: return tile<6, 1>(o, p.splits, st);
    default: return tile<8, 1>(o, p.splits, st);
  }
}

template <typename T>
hipError_t rows_t(const T* x, int rows, int K, int kc, int8_t* codes, float* scale, hipStream_t st) {
  if (4 * kc <= 256) {
    q8_rows_kernel<T, 4><<<rows, 256, 0, st>>>(x, K, kc, 4 * kc, codes, scale);
  } else {
    // parts of 256 pieces at least, as many as the chip has room for
    const int parts = std::max(1, std::min((4 * kc + 255) / 256, 512 / rows)), per = (4 * kc + parts - 1) / parts;
    q8_rows_kernel<T, 16><<<dim3(rows, parts), 1024, 0, st>>>(x, K, kc, per, codes, scale);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t small(const T* a, int m, const int8_t* codes, const float* scale, int N, int K, int kc, float* out, hipStream_t st) {
  q8_small_kernel<T><<<(N + 15) / 16, 1024, 0, st>>>(a, codes, scale, m, N, K, kc, out);
  return hipGetLastError();
}
hipError_t launch_rows(int dtype, const void* x, int rows, int K, int kc, int8_t* codes, float* scale, hipStream_t st) {
  return dtype == kBF16 ? rows_t((const bf16*)x, rows, K, kc, codes, scale, st) : rows_t((const float*)x, rows, K, kc, codes, scale, st);
}

}  // namespace

size_t q8_linear_bytes(int max_rows, int max_k) {
  return up256((size_t)(max_rows + 15) / 16 * 16 * ((q8_kpad(max_k) + 255) & ~255)) + up256((size_t)max_rows * 4) + kPartBytes;
}

hipError_t launch_q8_pack(int dtype, const void* w, int N, int K, int8_t* codes, float* scale, hipStream_t st) {
  return launch_rows(dtype, w, N, K, q8_kpad(K) / 64, codes, scale, st);
}

Q8LinearPlan q8_plan_linear(int m, int N, int K) {
  const int kc = q8_kpad(K) / 64, ka = (kc + 3) & ~3, m_tiles = (m + 15) / 16, n_tiles = (N + 15) / 16;
  // One launch; every workgroup rounds the rows again, so only up to three workgroups for two compute units.  In a captured loop of calls, us, one
  // launch and two: 5 x 768 x 256 3.9 and 5.4, 16 x 4096 x 1024 5.5 and 6.9, 16 x 4096 x 2048 7.2 and 8.1, 16 x 6144 x 1024 7.2 and 7.4,
  // 16 x 8192 x 2048 10.3 and 9.5 (two tiles of rows in one launch: 32 x 768 x 256 6.1 and 6.4, 32 x 2048 x 1024 7.2 and 6.8).
  if (m_tiles == 1 && kc <= 32 && n_tiles <= 384) return Q8LinearPlan{kQ8Small, 1, 1, 16, 1};
  // Up to two tiles of rows the activations come along from the L2 without weighing (a call of 1 x 3584 x 18944 18.3 us, through tiles
  // 19.9; 31 x 4096 x 12288 18.2 and 19.0); from three on a compute unit pulls more of them than of weights (37 x 3584 x 18944 25.4 and
  // 23.3, 63 x 12288 x 4096 21.2 and 17.6).
  if (m <= kStreamRows) {
    // Two column tiles a workgroup where that leaves a workgroup for each compute unit (2 x 12288 x 4096 15.1 us, with one 15.9, 18 x 14851
    // x 984 11.0 and 12.5; 31 x 4096 x 12288 22.6, with one 18.2)
    const int nt = n_tiles >= 512 ? 2 : 1, waves = nt == 2 ? 8 : 16;
    return Q8LinearPlan{kQ8Stream, m_tiles, nt, waves, plan_stream(m, N, kc, nt, waves)};
  }
  return plan_tile(m, N, ka);
}

hipError_t launch_q8_linear(int dtype, const void* a, int m, const int8_t* codes, const float* scale, int N, int K, float* out,
                            void* ws, hipStream_t st) {
  const int kc = q8_kpad(K) / 64, ka = (kc + 3) & ~3, m_tiles = (m + 15) / 16;
  const Q8LinearPlan plan = q8_plan_linear(m, N, K);
  if (plan.kernel == kQ8Small)
    return dtype == kBF16 ? small((const bf16*)a, m, codes, scale, N, K, kc, out, st)
                          : small((const float*)a, m, codes, scale, N, K, kc, out, st);
  char* p = (char*)ws;
  int8_t* qa = (int8_t*)p;
  p += up256((size_t)m_tiles * 16 * ka * 64);
  float* sa = (float*)p;
  p += up256((size_t)m * 4);
  const hipError_t e = launch_rows(dtype, a, m, K, ka, qa, sa, st);
  if (e != hipSuccess) return e;
  const Operands o{qa, sa, codes, scale, m, N, kc, ka, out, (int*)p};
  if (plan.kernel == kQ8Tile) return run_tile(o, plan, st);
  if (plan.mt == 1) return plan.nt == 2 ? stream<1, 2, 8>(o, plan.splits, st) : stream<1, 1, 16>(o, plan.splits, st);
  return plan.nt == 2 ? stream<2, 2, 8>(o, plan.splits, st) : stream<2, 1, 16>(o, plan.splits, st);
}

}  // namespace d2c
