// Products in 8-bit integers: out[m, N] = (sum_k qa[m, k] qw[n, k]) sa[m] sw[n], exact sums in 32 bits.
//
// Both operands lie in the order in which the matrix cores take them (v_mfma_i32_16x16x64_i8): tiles of 16 rows x 64 of the
// contraction, 1 KB each, lane l's 16 bytes (row l % 16, contraction 16 (l / 16) ..) at 16 l; rows and contraction are padded with
// zeros to whole tiles.  Weights are brought into that order once (q8_pack_kernel), activations in a launch of their own in front of
// each product (q8_rows_kernel), with a scale per row.
#include <algorithm>

#include "q8.h"

namespace d2c {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Rows quantised by their largest magnitude; a row that holds a NaN or an infinity gets the scale NaN.  One workgroup per row, 16
// columns per thread at a time, which is one lane's piece of a tile.  Rows from n_rows on are padding: zeros, no scale.
template <typename T>
__global__ __launch_bounds__(256) void q8_rows_kernel(const T* x, int n_rows, int K, int8_t* codes, float* scale) {
  const int r = blockIdx.x, tid = threadIdx.x, kc = (K + 63) / 64;
  const T* row = x + (size_t)r * K;
  __shared__ float red[4];
  float amax = 0.f;
  bool bad = false;
  if (r < n_rows)
    for (int k = 8 * tid; k < K; k += 2048) {
      float v[8];
      if (K - k >= 8) q8_load8(row + k, v);
      else { q8_load4(row + k, v); v[4] = v[5] = v[6] = v[7] = 0.f; }       // float rows of 4 more
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = fabsf(v[j]);
        bad |= !(a <= 3.402823466e38f);
        amax = fmaxf(amax, a);
      }
    }
  amax = wave_max(bad ? INFINITY : amax);
  if ((tid & 63) == 0) red[tid >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const bool nan_row = amax == INFINITY;
  const float s = nan_row ? 0.f : q8_scale(amax), inv = q8_inverse(s);
  if (tid == 0 && r < n_rows) scale[r] = nan_row ? __builtin_nanf("") : s;
  int8_t* to = codes + (size_t)(r / 16) * kc * 1024 + r % 16 * 16;
  for (int p = tid; p < 4 * kc; p += 256) {
    u32x4 w = {0, 0, 0, 0};
    if (r < n_rows && s > 0.f)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = 16 * p + 8 * half;
        float v[8] = {};
        if (K - k >= 8) q8_load8(row + k, v);
        else if (K - k >= 4) q8_load4(row + k, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[2 * half + j / 4] |= (uint32_t)(uint8_t)q8_code(v[j], s, inv) << (8 * (j % 4));
      }
    *reinterpret_cast<u32x4*>(to + (size_t)(p / 4) * 1024 + p % 4 * 256) = w;
  }
}

__device__ __forceinline__ i32x4 mfma_i8(const u32x4& a, const u32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// 16 outputs x MT tiles of 16 rows per workgroup; its four waves take every fourth step of the contraction.
template <int MT>
__global__ __launch_bounds__(256) void q8_linear_kernel(const int8_t* a, const float* sa, const int8_t* w, const float* sw, int m, int N,
                                                        int kc, float* out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_tile = blockIdx.x, m0 = blockIdx.y * MT, m_tiles = (m + 15) / 16;
  i32x4 acc[MT] = {};
  const int8_t* wp = w + (size_t)n_tile * kc * 1024 + lane * 16;
  for (int k = wave; k < kc; k += 4) {
    const u32x4 wf = ld16(wp + (size_t)k * 1024);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int mt = min(m0 + t, m_tiles - 1);
      acc[t] = mfma_i8(wf, ld16(a + ((size_t)mt * kc + k) * 1024 + lane * 16), acc[t]);
    }
  }
  __shared__ i32x4 red[3][MT][64];
#pragma unroll
  for (int t = 0; t < MT; ++t)
    if (wave) red[wave - 1][t][lane] = acc[t];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const i32x4 v = acc[t] + red[0][t][lane] + red[1][t][lane] + red[2][t][lane];
    const int row = (m0 + t) * 16 + lane % 16, n = n_tile * 16 + lane / 16 * 4;
    if (row < m)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < N) out[(size_t)row * N + n + j] = (float)v[j] * sa[row] * sw[n + j];
  }
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t q8_linear_bytes(int max_rows, int max_k, int max_n) {
  (void)max_n;
  return up256((size_t)(max_rows + 15) / 16 * 16 * q8_kpad(max_k)) + up256((size_t)max_rows * 4);
}

hipError_t launch_q8_rows(int dtype, const void* x, int rows, int padded, int K, int8_t* codes, float* scale, hipStream_t st) {
  if (dtype == kBF16) q8_rows_kernel<bf16><<<padded, 256, 0, st>>>((const bf16*)x, rows, K, codes, scale);
  else q8_rows_kernel<float><<<padded, 256, 0, st>>>((const float*)x, rows, K, codes, scale);
  return hipGetLastError();
}

hipError_t launch_q8_pack(int dtype, const void* w, int N, int K, int8_t* codes, float* scale, hipStream_t st) {
  return launch_q8_rows(dtype, w, N, (N + 15) / 16 * 16, K, codes, scale, st);
}

hipError_t launch_q8_linear(int dtype, const void* a, int m, const int8_t* codes, const float* scale, int N, int K, float* out,
                            void* ws, hipStream_t st) {
  const int kc = q8_kpad(K) / 64, m_tiles = (m + 15) / 16;
  int8_t* qa = (int8_t*)ws;
  float* sa = (float*)((char*)ws + up256((size_t)m_tiles * 16 * kc * 64));
  hipError_t e = launch_q8_rows(dtype, a, m, m_tiles * 16, K, qa, sa, st);
  if (e != hipSuccess) return e;
  const int n_tiles = (N + 15) / 16;
  if (m_tiles == 1) q8_linear_kernel<1><<<dim3(n_tiles, 1), 256, 0, st>>>(qa, sa, codes, scale, m, N, kc, out);
  else if (m_tiles == 2) q8_linear_kernel<2><<<dim3(n_tiles, 1), 256, 0, st>>>(qa, sa, codes, scale, m, N, kc, out);
  else q8_linear_kernel<4><<<dim3(n_tiles, (m_tiles + 3) / 4), 256, 0, st>>>(qa, sa, codes, scale, m, N, kc, out);
  return hipGetLastError();
}

}  // namespace d2c
