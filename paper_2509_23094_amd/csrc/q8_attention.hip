// Attention of a few query rows against a whole K/V cache held in 8 bits.
//
// A workgroup takes 32 query rows of one kv head (with grouped heads: rows of all its query heads) and a range of the cache's 64-row
// blocks, eight waves one block each at a time.  A wave forms S^T[64 keys x 32 rows] = K Q^T, its softmax terms, and
// O^T[D x 32 rows] += V^T P^T, all in registers: an accumulator of S^T holds, for one query row, the keys 8a + 4g + j (g = lane / 32),
// and V's codes lie in the cache as four rows of four dimensions, so that they are the other operand in just that order.
//   codes -> fp16 exactly: a byte u under the high byte 0x64 is the fp16 number 1024 + u, less 1152 gives code = u - 128 (one byte
//   permutation and one packed addition for two codes).  q enters as fp16 too: a row is scaled by a power of two so that its largest
//   magnitude lies in [2^14, 2^15).  bf16's 8 bits fit in whole down to 2^-32 of the largest (below: to the nearest 2^-39 of it);
//   float takes two pieces of 11 bits, which leave 2^-23 of each value and 2^-39 of the largest.  The product's scale (row, block and
//   log2(e) / sqrt(D)) is applied to the fp32 score, V's scale when a block's O^T joins the running one.
//   probabilities are rounded to fp16 (float: two pieces): 11 (22) bits down to 2^-25 (2^-18) of a row's largest, below that to
//   the nearest 2^-35 (2^-39) of it; the running sum takes them before that rounding.
// The waves' maxima, sums and O^T are merged through LDS; where the key range is split over workgroups, by a second launch.
// The head average has a pass of its own over the scores, from the same fp16 q and the final (maximum, sum) of every row.
#include <algorithm>
#include <cmath>

#include "q8.h"

namespace d2c {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 32;                 // query rows per workgroup
constexpr int kWaves = 8;
// Probabilities are rounded to fp16 relative to a reference that a score may pass by `slack`, times a power of two that takes them to 2^15 at most.
// bf16: 2^11 in the exponent, and a reference that is seldom raised.  Float, whose second piece would be a subnormal number sooner,
// keeps the four bits and multiplies by 2^15 behind the exponential, whose argument stays small (near 15 its rounding alone is 2^-21).
template <int QP> struct Base {
  static constexpr float bits = QP == 1 ? 11.f : 0.f, times = QP == 1 ? 1.f : 0x1p15f, slack = QP == 1 ? 4.f : 0.f;
  static constexpr float unit = QP == 1 ? 0x1p-11f : 1.f;       // 2^-bits
};

// log2(e) / sqrt(D)
template <int D> constexpr float kScore = 1.4426950408889634f / (D == 128 ? 11.313708498984761f : 8.f);

struct AttendSeq {
  Q8CachePtr c;
  const void* q;
  void* out;
  float* avg;
  int m, L;
  int splits, per_split;                  // workgroups over the keys, blocks of each
  int first_wg;                           // of the forward launch
  int row0;                               // first (row, head) slot in the workspace
  int avg_tiles, avg_first_wg;            // 32-row tiles of one head; first workgroup of the average's launch
  size_t q16;                             // this sequence's fp16 rows in the workspace, halves
};
struct AttendArgs {
  AttendSeq s[kQ8Launch];
  int n, H, Hkv;
  float* part;                            // [split][slot][D]
  float2* ml;                             // [split][slot]: maximum (base 2), sum
  _Float16* q16;
  f32x4* row;                             // [slot]: 1 / (power of two on the row), its reference, 1 / its sum of exponentials
  size_t slots;                           // of the whole launch
};

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// two codes of a word as fp16: bytes 2i and 2i + 1
__device__ __forceinline__ h2 codes2(uint32_t w, uint32_t sel) {
  const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w, sel);
  return __builtin_bit_cast(h2, u) + h2{(_Float16)-1152.f, (_Float16)-1152.f};
}
__device__ __forceinline__ h8 codes8(uint32_t a, uint32_t b) {
  const h2 x = codes2(a, 0x04010400u), y = codes2(a, 0x04030402u), z = codes2(b, 0x04010400u), w = codes2(b, 0x04030402u);
  return h8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

__device__ __forceinline__ f32x16 mfma(const h8& a, const h8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// the power of two that brings amax into [2^14, 2^15); 1 for 0 and what is not finite
__device__ __forceinline__ float pow2_for(float amax) {
  if (!(amax > 0.f) || !(amax <= 3.402823466e38f)) return 1.f;
  return ldexpf(1.f, max(-126, min(126, 14 - ilogbf(amax))));
}

// D / 16 operands of one query row half (16 dimensions of each 32), scaled; returns the scale
template <typename T, int D, int QP>
__device__ __forceinline__ float load_q(const T* q, h8 (&f)[QP][D / 16]) {
  float x[D / 2], amax = 0.f;
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    q8_load8(q + 32 * c + 16 * g, &x[16 * c]);
    q8_load8(q + 32 * c + 16 * g + 8, &x[16 * c + 8]);
  }
#pragma unroll
  for (int j = 0; j < D / 2; ++j) amax = fmaxf(amax, fabsf(x[j]));
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  const float p2 = pow2_for(amax);
#pragma unroll
  for (int j = 0; j < D / 2; ++j) {
    const float v = x[j] * p2;
    const _Float16 hi = (_Float16)v;
    f[0][j / 8][j % 8] = hi;
    if constexpr (QP > 1) f[1][j / 8][j % 8] = (_Float16)(v - (float)hi);
  }
  return p2;
}

// Operands of 32 keys: raw[c] = 16 dimensions of this lane's key in chunk 2c + g
template <int D>
__device__ __forceinline__ void convert_k(const u32x4 (&raw)[D / 32], h8 (&k)[D / 16]) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    k[2 * c] = codes8(raw[c][0], raw[c][1]);
    k[2 * c + 1] = codes8(raw[c][2], raw[c][3]);
  }
}
// S^T of 32 keys
template <int D, int QP>
__device__ __forceinline__ f32x16 product(const h8 (&k)[D / 16], const h8 (&q)[QP][D / 16]) {
  f32x16 acc = {};
#pragma unroll
  for (int f = 0; f < D / 16; ++f)
#pragma unroll
    for (int p = 0; p < QP; ++p) acc = mfma(k[f], q[p][f], acc);
  return acc;
}
template <int D, int QP>
__device__ __forceinline__ f32x16 scores(const u32x4 (&raw)[D / 32], const h8 (&q)[QP][D / 16]) {
  h8 k[D / 16];
  convert_k<D>(raw, k);
  return product<D, QP>(k, q);
}
template <int D>
__device__ __forceinline__ void load_k(const uint8_t* k, int key, u32x4 (&raw)[D / 32]) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) raw[c] = ld16(k + (2 * c + g) * 1024 + key * 16);
}

// Pieces of V of a block: eight times four rows of this lane's D / 32 dimensions (D = 64: eight bytes of each)
template <int D>
__device__ __forceinline__ void load_v(const uint8_t* v, u32x4 (&raw)[8]) {
  const int g = (threadIdx.x & 63) >> 5, r32 = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint8_t* at = v + (2 * i + g) * 4 * D + r32 * (D / 8);
    if constexpr (D == 128) raw[i] = ld16(at);
    else { const u32x2 w = ld8(at); raw[i][0] = w[0]; raw[i][1] = w[1]; }
  }
}

// Scores of a block (`left` of its keys exist) -> probabilities in operand order.  o and l are relative to 2^ref; ref is raised only where
// a score passes it by more than the slack.
template <int QP, int DT>
__device__ __forceinline__ void softmax_step(f32x16 (&x)[2], float ks, int left, float& ref, float& l, f32x16 (&o)[DT], h8 (&p)[QP][4]) {
  constexpr float kSlack = Base<QP>::slack;
  const int g = (threadIdx.x & 63) >> 5;
  float top = -3.4e38f;
  if (left >= kQ8Rows) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
  } else {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * t + 8 * (i / 4) + 4 * g + i % 4 < left) top = fmaxf(top, x[t][i]);
  }
  top = fmaxf(top, __shfl_xor(top, 32, 64)) * ks;
  if (__any(top > ref + kSlack)) {
    const float to = top > ref + kSlack ? top : ref, alpha = exp2_hw(ref - to);
    ref = to;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
  }
  const float base = Base<QP>::bits - ref;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[t][i] = exp2_hw(fmaf(x[t][i], ks, base));
  if (left < kQ8Rows) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * t + 8 * (i / 4) + 4 * g + i % 4 >= left) x[t][i] = 0.f;
  }
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sum += x[t][i];
      const _Float16 hi = (_Float16)(x[t][i] * Base<QP>::times);
      p[0][2 * t + i / 8][i % 8] = hi;
      if constexpr (QP > 1) p[1][2 * t + i / 8][i % 8] = (_Float16)fmaf(x[t][i], Base<QP>::times, -(float)hi);
    }
  l += sum;
}

// One tile of rows per workgroup: its waves take blocks in turn, operands straight from memory.
// What bounds it: a wave's chain through a block, keys -> scores -> maximum -> exponentials -> values, which the two waves per SIMD that the
// registers allow do not hide, and 5 us at its ends.  28 heads on 4, 19 rows x 60001 keys: vector units busy 72 % of the time, matrix cores 29 %, waves
// waiting 32 %, with 571 vector instructions per wave and block (256 of them to make fp16 of codes); 32 heads, 256 x 2048, where the ends weigh more, 64,
// 22 and 31 %.  Times: 36 us, 18-20 us, 4 sequences of up to 45 rows x 1823 keys 18.7 us (their 192 workgroups have 29 to 13 blocks
// each and all wait for the longest); float 256 x 2048 29 us.  Of D = 128 bf16 spills 2 registers around the loop, float 10, one of which is
// loaded again for each block.  Tried without gain: codes shared in LDS by the tiles of rows, keys requested two blocks
// ahead, priorities for half the waves.  Codes left 1152 too large, with the sums put right afterwards, is a fifth fewer vector instructions,
// 2-6 % faster, and loses up to 2^-12 of a step of the codes: not kept.
template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void q8_attend_kernel(AttendArgs args) {
  constexpr int QP = sizeof(T) == 2 ? 1 : 2;      // fp16 pieces of q and of a probability
  constexpr int DT = D / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, r32 = lane & 31;
  int si = 0;
  while (si + 1 < args.n && (int)blockIdx.x >= args.s[si + 1].first_wg) ++si;
  const AttendSeq& s = args.s[si];
  // (kv head, split) runs fastest: the row tiles that read the same keys are 8 k workgroups apart, on one XCD
  const int local = blockIdx.x - s.first_wg, groups = args.Hkv * s.splits;
  const int hk = local % groups % args.Hkv, split = local % groups / args.Hkv, tile = local / groups;
  const int G = args.H / args.Hkv, R = s.m * G, n_blocks = (s.L + kQ8Rows - 1) / kQ8Rows;
  const int b0 = split * s.per_split, b1 = min(n_blocks, b0 + s.per_split);
  const int r = tile * kTile + r32;
  const bool valid = r < R;                        // past the last: the first row again, not stored
  const int row = valid ? r / G : 0, head = hk * G + (valid ? r % G : 0);

  u32x4 kr[2][D / 32], vr[8];
  float ks_next, vs_next;
  // the next block's keys are requested as soon as this block's are used (float, whose q takes twice the registers: when they are
  // needed), its values likewise; behind the last block that one again
  auto want_k = [&](int b) __attribute__((always_inline)) {
    const size_t blk = (size_t)min(b, b1 - 1) * args.Hkv + hk;
    load_k<D>(s.c.k + blk * kQ8Rows * D, r32, kr[0]);
    load_k<D>(s.c.k + blk * kQ8Rows * D, 32 + r32, kr[1]);
    ks_next = s.c.ks[blk];
  };
  auto want_v = [&](int b) __attribute__((always_inline)) {
    const size_t blk = (size_t)min(b, b1 - 1) * args.Hkv + hk;
    load_v<D>(s.c.v + blk * kQ8Rows * D, vr);
    vs_next = s.c.vs[blk];
  };
  if (QP == 1) want_k(b0 + wave);
  want_v(b0 + wave);
  h8 q[QP][D / 16];
  const float p2 = load_q<T, D, QP>((const T*)s.q + ((size_t)row * args.H + head) * D, q);
  // a block's scores take ks * kScore * rp2, in this order: the row's power of two alone can be near the ends of the range (2^126 on tiny rows)
  const float rp2 = 1.f / p2;
  if (s.avg && split == 0 && wave == 0 && valid) {
    _Float16* to = args.q16 + s.q16 + (((size_t)head * s.avg_tiles + row / kTile) * (QP * D / 16) * 64 + g * 32 + row % kTile) * 8;
#pragma unroll
    for (int p = 0; p < QP; ++p)
#pragma unroll
      for (int f = 0; f < D / 16; ++f) *reinterpret_cast<h8*>(to + (size_t)(p * (D / 16) + f) * 512) = q[p][f];
  }

  f32x16 o[DT] = {};
  float ref = -INFINITY, l = 0.f;
  for (int b = b0 + wave; b < b1; b += kWaves) {
    if (QP > 1) want_k(b);
    const float ks = ks_next * kScore<D> * rp2;
    f32x16 x[2];
    x[0] = scores<D, QP>(kr[0], q);
    x[1] = scores<D, QP>(kr[1], q);
    if (QP == 1) want_k(b + kWaves);
    h8 p[QP][4];
    softmax_step<QP, DT>(x, ks, s.L - b * kQ8Rows, ref, l, o, p);
    const float vs = vs_next * (1.f / Base<QP>::times);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f32x16 acc = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const h8 a = codes8(vr[2 * i][dt], vr[2 * i + 1][dt]);
#pragma unroll
        for (int pp = 0; pp < QP; ++pp) acc = mfma(a, p[pp][i], acc);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = fmaf(vs, acc[i], o[dt][i]);
    }
    want_v(b + kWaves);
  }
  l += __shfl_xor(l, 32, 64);

  // merge the waves: each adds up an eighth of every accumulator, two times D / 32 neighbouring dimensions of a row
  __shared__ float lds[kWaves][DT * 16][64];
  __shared__ float wref[kWaves][kTile], wl[kWaves][kTile];
  if (g == 0) { wref[wave][r32] = ref; wl[wave][r32] = l; }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) lds[wave][dt * 16 + i][lane] = o[dt][i];
  __syncthreads();
  if (!valid) return;
  float M = wref[0][r32], sum = 0.f, weight[kWaves];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, wref[w][r32]);
  const float to_m = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    weight[w] = exp2_hw(wref[w][r32] - to_m);
    sum += wl[w][r32] * weight[w];
  }
  float y[2 * DT];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) t = fmaf(lds[w][dt * 16 + 2 * wave + j][lane], weight[w], t);
      y[j * DT + dt] = t;
    }
  // row 8 (wave / 2) + 4 g + 2 (wave % 2) + j of tile dt is dimension DT * (that) + dt
  const int d0 = (wave / 2 * 8 + 4 * g + wave % 2 * 2) * DT;
  const size_t slot = (size_t)s.row0 + (size_t)row * args.H + head;
  if (s.splits > 1) {
    float* to = args.part + ((size_t)split * args.slots + slot) * D + d0;
#pragma unroll
    for (int j = 0; j < DT / 2; ++j) q8_store4(to + 4 * j, y + 4 * j);
    if (wave == 0 && g == 0) args.ml[(size_t)split * args.slots + slot] = make_float2(M, sum);
  } else {
    const float inv = 1.f / sum;
#pragma unroll
    for (int j = 0; j < 2 * DT; ++j) y[j] *= inv;
    T* to = (T*)s.out + ((size_t)row * args.H + head) * D + d0;
#pragma unroll
    for (int j = 0; j < DT / 2; ++j) q8_store4(to + 4 * j, y + 4 * j);
  }
  if (s.avg && wave == 0 && g == 0 && split == 0)
    args.row[slot] = f32x4{rp2, to_m, 1.f / (sum * Base<QP>::unit), 0.f};      // (of a split row: the merge puts it right)
}

// Splits of a row joined.  A workgroup per row and head, a thread per (four dimensions, every kJoin-th split).  What bounds it: launching and
// one latency; 19 rows x 28 heads of 12 splits 5.2 us.
constexpr int kJoin = 8;
template <typename T, int D>
__global__ __launch_bounds__(kJoin * D / 4) void q8_join_kernel(AttendArgs args) {
  const int t = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
  const size_t slot = blockIdx.x;
  int si = 0;
  while (si + 1 < args.n && slot >= (size_t)args.s[si + 1].row0) ++si;
  const AttendSeq& s = args.s[si];
  if (s.splits <= 1) return;
  float M = -INFINITY, sum = 0.f;
  f32x4 y = {};
  for (int i = part; i < s.splits; i += kJoin) {
    const float2 ml = args.ml[(size_t)i * args.slots + slot];
    const f32x4 z = *reinterpret_cast<const f32x4*>(args.part + ((size_t)i * args.slots + slot) * D + 4 * t);
    const float m = fmaxf(M, ml.x), ref = m == -INFINITY ? 0.f : m, a = exp2_hw(M - ref), w = exp2_hw(ml.x - ref);
    M = m;
    sum = sum * a + ml.y * w;
    y = y * a + z * w;
  }
  __shared__ float sm[kJoin], ss[kJoin];
  __shared__ f32x4 sy[kJoin][D / 4];
  if (t == 0) { sm[part] = M; ss[part] = sum; }
  sy[part][t] = y;
  __syncthreads();
  if (part) return;
#pragma unroll
  for (int i = 1; i < kJoin; ++i) M = fmaxf(M, sm[i]);
  const float ref = M == -INFINITY ? 0.f : M;
  sum = 0.f;
  y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kJoin; ++i) {
    const float w = exp2_hw(sm[i] - ref);
    sum += ss[i] * w;
    y += sy[i][t] * w;
  }
  y *= 1.f / sum;
  float z[4] = {y[0], y[1], y[2], y[3]};
  q8_store4((T*)s.out + (slot - s.row0) * D + 4 * t, z);
  if (s.avg && t == 0) {
    args.row[slot][1] = ref;
    args.row[slot][2] = 1.f / (sum * Base<sizeof(T) == 2 ? 1 : 2>::unit);
  }
}

// attn_avg of 32 rows x one block of keys: the waves take a run of heads each and are added up at the end.  The next head's keys and
// queries are on their way while one head's are used.  What bounds it: the same chain without the values: vector units busy 44 % of the
// time, matrix cores 18 %, waves waiting 40 % (32 heads, 256 rows x 2048 keys, 11.7 us; a compute unit gets 45 KB/us of codes and queries from
// its L2).  4 sequences of up to 45 x 1823 12.4 us.
template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void q8_average_kernel(AttendArgs args) {
  constexpr int QP = sizeof(T) == 2 ? 1 : 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, r32 = lane & 31;
  int si = 0;
  while (si + 1 < args.n && (int)blockIdx.x >= args.s[si + 1].avg_first_wg) ++si;
  const AttendSeq& s = args.s[si];
  const int n_blocks = (s.L + kQ8Rows - 1) / kQ8Rows, local = blockIdx.x - s.avg_first_wg;
  const int b = local % n_blocks, tile = local / n_blocks, row = min(tile * kTile + r32, s.m - 1), G = args.H / args.Hkv;
  const int h0 = wave * args.H / kWaves, h1 = (wave + 1) * args.H / kWaves;
  f32x16 acc[2] = {};
  u32x4 kr[2][D / 32];
  h8 k[2][D / 16], q[QP][D / 16];
  f32x4 rw = {};
  float ks_next = 0.f, ks = 0.f;
  auto want_k = [&](int hk) __attribute__((always_inline)) {
    const size_t blk = (size_t)b * args.Hkv + hk;
    load_k<D>(s.c.k + blk * kQ8Rows * D, r32, kr[0]);
    load_k<D>(s.c.k + blk * kQ8Rows * D, 32 + r32, kr[1]);
    ks_next = s.c.ks[blk];
  };
  auto want_q = [&](int h) __attribute__((always_inline)) {
    const _Float16* from = args.q16 + s.q16 + (((size_t)h * s.avg_tiles + tile) * (QP * D / 16) * 64 + lane) * 8;
#pragma unroll
    for (int p = 0; p < QP; ++p)
#pragma unroll
      for (int f = 0; f < D / 16; ++f) q[p][f] = __builtin_bit_cast(h8, ld16(from + (size_t)(p * (D / 16) + f) * 512));
    rw = args.row[(size_t)s.row0 + (size_t)row * args.H + h];
  };
  if (h0 < h1) {
    want_k(h0 / G);
    want_q(h0);
  }
  for (int h = h0; h < h1; ++h) {
    if (h == h0 || h % G == 0) {                     // the heads of a kv head share its operands
      convert_k<D>(kr[0], k[0]);
      convert_k<D>(kr[1], k[1]);
      ks = ks_next;
      want_k(min(h / G + 1, args.Hkv - 1));
    }
    const float c = ks * kScore<D> * rw[0], base = -rw[1], inv = rw[2];
    f32x16 x[2];
    x[0] = product<D, QP>(k[0], q);
    x[1] = product<D, QP>(k[1], q);
    want_q(min(h + 1, h1 - 1));
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = fmaf(exp2_hw(fmaf(x[t][i], c, base)), inv, acc[t][i]);
  }
  __shared__ float lds[kWaves][kTile][kQ8Rows + 1];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) lds[wave][r32][32 * t + 8 * (i / 4) + 4 * g + i % 4] = acc[t][i];
  __syncthreads();
  const int key = b * kQ8Rows + lane;
  if (key >= s.L) return;
  const float inv = 1.f / args.H;
#pragma unroll
  for (int i = 0; i < kTile / kWaves; ++i) {
    const int rr = kWaves * i + wave, at = tile * kTile + rr;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += lds[w][rr][lane];
    if (at < s.m) s.avg[(size_t)at * s.L + key] = sum * inv;
  }
}

// Workgroups over the keys, by an estimate of the time in us, fitted to 144 cases (1-512 rows, 64-65536 keys, one to five sequences, all numbers
// of splits measured on each; what it picks is 0.9 % behind the best on average, 8 % at most).  A compute unit holds one workgroup; a round
// over eight blocks takes it 2.5, over fewer less, its ends 5; a split row takes a launch and its way to memory and back.
// 28 heads on 4, bf16, 1 row x 1023 keys: unsplit 11.3 us, 8 splits 9.7; 19 rows x 60001 unsplit 273, 12 splits 37.
constexpr int kTargetWgs = 512;
int plan_splits(int workgroups, int most_blocks) {
  constexpr float round = 2.5f, fixed = 0.28f, ends = 5.f, join = 2.6f, each = 0.0059f;
  int best = 1;
  float best_cost = 1e30f;
  for (int s = 1; s <= 64 && (s == 1 || (s * workgroups <= kTargetWgs && 2 * s <= most_blocks)); ++s) {
    const int blocks = (most_blocks + s - 1) / s, rest = blocks % kWaves;
    const float rounds = blocks / kWaves + (rest ? fixed + (1.f - fixed) * rest / kWaves : 0.f);
    const float cost = (s * workgroups + 255) / 256 * (round * rounds + ends) + (s > 1 ? join + s * workgroups * each : 0.f);
    if (cost < best_cost) { best_cost = cost; best = s; }
  }
  return best;
}
int row_tiles(const Q8Shape& s, int m) { return (m * (s.H / s.Hkv) + kTile - 1) / kTile; }

// Workspace: partial sums of split rows -- splits x rows is at most kTargetWgs tiles, as rows are at most 32 per unsplit
// workgroup -- and, for the average, the softmax's numbers and fp16 rows of every query row and head.
struct Layout { size_t ml, row, q16, total; };
Layout layout(const Q8Shape& s, size_t max_rows, size_t max_batch) {
  const size_t split_rows = (size_t)kTargetWgs * kTile, pieces = s.dtype == kBF16 ? 1 : 2;
  const size_t q_rows = max_rows + (kTile - 1) * std::min<size_t>(max_batch, kQ8Launch);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  Layout l;
  l.ml = up(split_rows * s.D * 4);
  l.row = l.ml + up(split_rows * 8);
  l.q16 = l.row + up(max_rows * s.H * 16);
  l.total = l.q16 + up(q_rows * s.H * pieces * s.D * 2);
  return l;
}

template <typename T, int D>
hipError_t run(const AttendArgs& a, int wgs, int avg_wgs, bool join, hipStream_t st) {
  q8_attend_kernel<T, D><<<wgs, 64 * kWaves, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && join) {
    q8_join_kernel<T, D><<<(unsigned)a.slots, kJoin * D / 4, 0, st>>>(a);
    e = hipGetLastError();
  }
  if (e == hipSuccess && avg_wgs) {
    q8_average_kernel<T, D><<<avg_wgs, 64 * kWaves, 0, st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t q8_attention_bytes(const Q8Shape& s, int max_rows, int max_batch) { return layout(s, max_rows, max_batch).total; }

hipError_t launch_q8_attention(const Q8Shape& s, const Q8Attend* calls, int n, int max_rows, int max_batch, void* ws, hipStream_t st) {
  const Layout l = layout(s, max_rows, max_batch);
  const int pieces = s.dtype == kBF16 ? 1 : 2;
  for (int c0 = 0; c0 < n; c0 += kQ8Launch) {
    AttendArgs a{};
    a.n = std::min(kQ8Launch, n - c0);
    a.H = s.H;
    a.Hkv = s.Hkv;
    a.part = (float*)ws;
    a.ml = (float2*)((char*)ws + l.ml);
    a.row = (f32x4*)((char*)ws + l.row);
    a.q16 = (_Float16*)((char*)ws + l.q16);
    int base = 0, most = 0, wgs = 0, avg_wgs = 0;
    size_t rows = 0;
    bool join = false;
    for (int i = 0; i < a.n; ++i) {
      base += row_tiles(s, calls[c0 + i].m) * s.Hkv;
      most = std::max(most, q8_blocks(calls[c0 + i].L));
    }
    const int splits = plan_splits(base, most);
    for (int i = 0; i < a.n; ++i) {
      const Q8Attend& c = calls[c0 + i];
      AttendSeq& q = a.s[i];
      const int nb = q8_blocks(c.L);
      q.c = c.cache; q.q = c.q; q.out = c.out; q.avg = c.avg; q.m = c.m; q.L = c.L;
      q.splits = std::min(splits, nb);
      q.per_split = (nb + q.splits - 1) / q.splits;
      q.splits = (nb + q.per_split - 1) / q.per_split;      // none empty
      q.first_wg = wgs;
      wgs += row_tiles(s, c.m) * s.Hkv * q.splits;
      q.row0 = (int)a.slots;
      a.slots += (size_t)c.m * s.H;
      q.avg_tiles = (c.m + kTile - 1) / kTile;
      q.avg_first_wg = avg_wgs;
      if (c.avg) avg_wgs += q.avg_tiles * nb;
      q.q16 = rows * s.H * pieces * s.D;
      rows += (size_t)q.avg_tiles * kTile;
      join = join || q.splits > 1;
    }
    const hipError_t e = s.dtype == kBF16 ? (s.D == 128 ? run<bf16, 128>(a, wgs, avg_wgs, join, st) : run<bf16, 64>(a, wgs, avg_wgs, join, st))
                                          : (s.D == 128 ? run<float, 128>(a, wgs, avg_wgs, join, st) : run<float, 64>(a, wgs, avg_wgs, join, st));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace d2c
