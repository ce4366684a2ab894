// Launch interface of the 8-bit operators' kernels (see include/d2c_q8.h), and what their device code shares.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "internal.h"

namespace d2c {

constexpr int kQ8Rows = 64;                   // cache rows per block (and scale)
constexpr int kQ8Launch = 8;                  // sequences of one launch: their descriptions are kernel arguments
inline int q8_blocks(int64_t rows) { return (int)((rows + kQ8Rows - 1) / kQ8Rows); }

struct Q8Shape { int H, Hkv, D, dtype; };
struct Q8CachePtr { uint8_t *k, *v; float *ks, *vs; };

struct Q8Update {
  Q8CachePtr cache;
  const int32_t* idx;
  const void *new_k, *new_v;
  int m, L;
};
hipError_t launch_q8_update(const Q8Shape& s, const Q8Update* calls, int n, hipStream_t st);
hipError_t launch_q8_read(const Q8Shape& s, const Q8CachePtr& cache, int L, const int32_t* idx, int n, void* out_k, void* out_v,
                          hipStream_t st);
hipError_t launch_q8_weigh(const float* avg, int m, int L, int64_t* weight, hipStream_t st);
hipError_t launch_q8_keep(const int64_t* weight, const uint8_t* protect, int L, int n_keep, int32_t* kept, int64_t* kept_weight,
                          hipStream_t st);
hipError_t launch_q8_compact(const Q8Shape& s, const Q8CachePtr& src, const int32_t* kept, int n_keep, const Q8CachePtr& dst,
                             hipStream_t st);

struct Q8Attend {
  Q8CachePtr cache;
  const void* q;
  void* out;
  float* avg;
  int m, L;
};
// bytes of workspace for calls of up to max_rows query rows in up to max_batch sequences
size_t q8_attention_bytes(const Q8Shape& s, int max_rows, int max_batch);
// calls with m > 0; max_rows and max_batch as the workspace was sized for
hipError_t launch_q8_attention(const Q8Shape& s, const Q8Attend* calls, int n, int max_rows, int max_batch, void* ws, hipStream_t st);

// How a product is launched: in one launch, or its rows rounded first and the product by weights streamed past few rows or by tiles
enum { kQ8Small = 0, kQ8Stream = 1, kQ8Tile = 2 };
struct Q8LinearPlan { int kernel, mt, nt, waves, splits; };   // row tiles per workgroup, column tiles per wave; waves of a workgroup, splits of the contraction
Q8LinearPlan q8_plan_linear(int m, int N, int K);
inline int q8_kpad(int K) { return (K + 63) & ~63; }
// bytes of workspace for products of up to max_rows rows and contractions of up to max_k
size_t q8_linear_bytes(int max_rows, int max_k);
hipError_t launch_q8_pack(int dtype, const void* w, int N, int K, int8_t* codes, float* scale, hipStream_t st);
hipError_t launch_q8_linear(int dtype, const void* a, int m, const int8_t* codes, const float* scale, int N, int K, float* out,
                            void* ws, hipStream_t st);

#ifdef __HIPCC__
// ---- quantising
__device__ __forceinline__ float q8_scale(float amax) { return amax < 0x1p-100f ? 0.f : amax / 127.f; }
__device__ __forceinline__ float q8_inverse(float s) { return s > 0.f ? 1.f / s : 0.f; }

// The whole number nearest to x / s (s > 0, inv about 1 / s), ties to even, in [-127, 127].  The product with inv can land on
// the wrong side of a border; the remainder x - n s tells, and has no rounding: it is a multiple of half of s's last place, and
// about s / 2 at most.  (Borders are not rare: half of a row's largest magnitude is one.)  No branches.
__device__ __forceinline__ int q8_code(float x, float s, float inv) {
  const float n = fminf(fmaxf(rintf(x * inv), -127.f), 127.f);
  const float e = fmaf(-n, s, x), e2 = 2.f * fabsf(e);
  const bool odd = (__builtin_bit_cast(uint32_t, n + 12582912.f) & 1u) != 0;
  const bool over = (e2 > s) | ((e2 == s) & odd);
  const float c = fminf(fmaxf(n + (over ? copysignf(1.f, e) : 0.f), -127.f), 127.f);
  return (x == x) & (s > 0.f) ? (int)c : 0;
}
// code(c * old, s): the product has 31 bits
__device__ __forceinline__ int q8_recode(int c, float old, float s, float inv) {
  const double x = (double)c * (double)old;
  const float n = fminf(fmaxf(rintf((float)x * inv), -127.f), 127.f);
  const double e = fma(-(double)n, (double)s, x), e2 = 2.0 * fabs(e);
  const bool odd = (__builtin_bit_cast(uint32_t, n + 12582912.f) & 1u) != 0;
  const bool over = (e2 > (double)s) | ((e2 == (double)s) & odd);
  const float r = fminf(fmaxf(n + (over ? copysignf(1.f, (float)e) : 0.f), -127.f), 127.f);
  return s > 0.f ? (int)r : 0;
}
// Sixteen codes at a time, as cache bytes.  The sum with 1.5 * 2^23 leaves the whole number nearest to x / s (or its neighbour, next to a
// border) in its low bits; the remainders say if all sixteen are the nearest: only where one is half a step or more (values that are
// not finite among them) is each done by itself.  byte[i]: code(x[i], s) + 128 in the low byte, other bits anything.
__device__ __forceinline__ void q8_bytes16(const float (&x)[16], float s, float inv, uint32_t (&byte)[16]) {
  constexpr float kMagic = 12582912.f + 128.f;
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float n = fmaf(x[i], inv, kMagic);
    worst = fmaxf(worst, fabsf(fmaf(-(n - kMagic), s, x[i])));
    byte[i] = __builtin_bit_cast(uint32_t, n);
    worst = fabsf(x[i]) <= 3.402823466e38f ? worst : INFINITY;
  }
  if (!(worst < 0.5f * s))
#pragma unroll
    for (int i = 0; i < 16; ++i) byte[i] = (uint32_t)(q8_code(x[i], s, inv) + 128);
}
// low bytes of four words in one
__device__ __forceinline__ uint32_t q8_pack(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// Four bytes of a word of old codes (scale old) as codes for s; inv about 1 / s, ratio about old / s.  The remainder in 32 bits is off by less than
// 1e-5 s (127 old 2^-24, old <= s): where one is that near to a border, all four are done in 64 bits.
__device__ __forceinline__ uint32_t q8_reword(uint32_t word, float old, float s, float inv, float ratio) {
  constexpr float kMagic = 12582912.f + 128.f;
  float worst = 0.f;
  uint32_t b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float c = (float)(word >> (8 * j) & 255u) - 128.f, n = fmaf(c, ratio, kMagic);
    worst = fmaxf(worst, fabsf(fmaf(-(n - kMagic), s, c * old)));
    b[j] = __builtin_bit_cast(uint32_t, n);
  }
  if (!(worst < 0.49998f * s))
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = (uint32_t)(q8_recode((int)(word >> (8 * j) & 255u) - 128, old, s, inv) + 128);
  return q8_pack(b[0], b[1], b[2], b[3]);
}
// eight neighbouring values of T as floats (16 bytes of bf16, 32 of float)
__device__ __forceinline__ void q8_load8(const bf16* p, float* x) {
  const bf16x8 v = __builtin_bit_cast(bf16x8, ld16(p));
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
}
__device__ __forceinline__ void q8_load8(const float* p, float* x) {
  const f32x4 a = __builtin_bit_cast(f32x4, ld16(p)), b = __builtin_bit_cast(f32x4, ld16(p + 4));
#pragma unroll
  for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
}
// four neighbouring values of T as floats
__device__ __forceinline__ void q8_load4(const bf16* p, float* x) {
  const bf16x4 v = __builtin_bit_cast(bf16x4, ld8(p));
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = (float)v[j];
}
__device__ __forceinline__ void q8_load4(const float* p, float* x) {
  const f32x4 v = __builtin_bit_cast(f32x4, ld16(p));
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = v[j];
}
__device__ __forceinline__ void q8_store4(bf16* p, const float* x) {
  bf16x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (bf16)x[j];
  *reinterpret_cast<u32x2*>(p) = __builtin_bit_cast(u32x2, v);
}
__device__ __forceinline__ void q8_store4(float* p, const float* x) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
}
__device__ __forceinline__ int q8_code_of(uint32_t word, int byte) { return (int)((word >> (8 * byte)) & 255u) - 128; }
#endif

}  // namespace d2c
