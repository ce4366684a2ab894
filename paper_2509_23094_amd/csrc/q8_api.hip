// C ABI of the 8-bit operators (see include/d2c_q8.h): argument validation, workspace and the order of kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <new>

#include "../../include/d2c_q8.h"
#include "../../include/d2c_tools.h"
#include "q8.h"

using namespace d2c;

constexpr int kMaxBatch = 256, kSeqBuffers = 10;

// A buffer of a call: where it lies, and what the call does with it.  Calls may read a cache that they refresh for another sequence.
enum Use { kReads, kWrites, kReadsCache, kRefreshes };
struct Range {
  uintptr_t at, end;
  Use use;
};

struct d2c_q8 {
  d2c_q8_dims dims{};
  Q8Shape shape{};
  int device = 0, max_batch = 1;
  void* ws = nullptr;            // shared by attention and linear: calls do not overlap
  int64_t ws_bytes = 0;
  Range ranges[kMaxBatch * kSeqBuffers];   // of the call that is checked
  int n_ranges = 0;
  char err[256] = {};
};

namespace {

thread_local char g_err[256] = {};     // of this thread's last d2c_q8_init

// Text without allocation: nothing here can throw.
int fail(d2c_q8* c, int code, const char* msg, const char* more = "") {
  snprintf(c ? c->err : g_err, 256, "%s%s", msg, more);
  return code;
}
int hip(d2c_q8* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return D2C_OK;
  (void)hipGetLastError();
  snprintf(c->err, sizeof c->err, "%s: %s", what, hipGetErrorString(e));
  return D2C_EHIP;
}

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

void add(d2c_q8* c, const void* p, size_t bytes, Use use) {
  if (p && bytes) c->ranges[c->n_ranges++] = Range{(uintptr_t)p, (uintptr_t)p + bytes, use};
}
void add_cache(d2c_q8* c, const d2c_q8_cache& k, int rows, Use use) {
  const size_t codes = (size_t)q8_blocks(rows) * c->dims.n_kv_heads * D2C_Q8_BLOCK * c->dims.head_dim;
  const size_t scales = (size_t)q8_blocks(rows) * c->dims.n_kv_heads * 4;
  add(c, k.k_codes, codes, use);
  add(c, k.v_codes, codes, use);
  add(c, k.k_scale, scales, use);
  add(c, k.v_scale, scales, use);
}
size_t row_bytes(const d2c_q8* c, int heads) { return (size_t)heads * c->dims.head_dim * (c->dims.dtype == D2C_BF16 ? 2 : 4); }
// What is written must not overlap anything else of the call.  In the order of their addresses a buffer overlaps one before it if that
// one, or any other of its use, ends behind its start.
int check_overlap(d2c_q8* c) {
  static constexpr bool kClash[4][4] = {{false, true, false, true}, {true, true, true, true}, {false, true, false, false}, {true, true, false, true}};
  std::sort(c->ranges, c->ranges + c->n_ranges, [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t end[4] = {};
  for (int i = 0; i < c->n_ranges; ++i) {
    const Range& r = c->ranges[i];
    for (int u = 0; u < 4; ++u)
      if (kClash[r.use][u] && end[u] > r.at)
        return fail(c, D2C_EINVAL, r.use == kRefreshes && u == kRefreshes ? "buffers of the caches that the call refreshes overlap"
                                                                          : "a buffer that the call writes overlaps another of its buffers");
    end[r.use] = std::max(end[r.use], r.end);
  }
  return D2C_OK;
}
Q8CachePtr ptr(const d2c_q8_cache& c) { return Q8CachePtr{c.k_codes, c.v_codes, c.k_scale, c.v_scale}; }

int check_device(d2c_q8* c) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(c, D2C_EHIP, "hipGetDevice failed");
  return dev == c->device ? D2C_OK : fail(c, D2C_EINVAL, "another device is current than the handle's");
}
int check_cache(d2c_q8* c, const d2c_q8_cache& k, int L) {
  if (c->dims.max_seq == 0) return fail(c, D2C_ESHAPE, "the handle was made without max_seq");
  if (L <= 0) return fail(c, D2C_EINVAL, "L must be positive");
  if (L > c->dims.max_seq) return fail(c, D2C_ESHAPE, "L exceeds max_seq of the handle");
  if (!k.k_codes || !k.v_codes || !k.k_scale || !k.v_scale) return fail(c, D2C_EINVAL, "null cache buffer");
  if (!aligned(k.k_codes, 16) || !aligned(k.v_codes, 16) || !aligned(k.k_scale, 4) || !aligned(k.v_scale, 4))
    return fail(c, D2C_EINVAL, "cache buffers must be aligned (codes to 16 bytes)");
  return D2C_OK;
}
// attend: the fields of d2c_q8_attention are looked at too
int check_seqs(d2c_q8* c, const d2c_q8_seq* seqs, int batch, bool attend) {
  if (batch < 0 || (batch > 0 && !seqs)) return fail(c, D2C_EINVAL, "bad batch");
  if (batch > c->max_batch) return fail(c, D2C_ESHAPE, "batch exceeds max_batch of the handle");
  int64_t rows = 0, tiles = 0;
  c->n_ranges = 0;
  for (int i = 0; i < batch; ++i) {
    const d2c_q8_seq& s = seqs[i];
    if (s.m < 0) return fail(c, D2C_EINVAL, "m must not be negative");
    if (s.m == 0) continue;
    int rc = check_cache(c, s.cache, s.L);
    if (rc) return rc;
    if ((s.new_k == nullptr) != (s.new_v == nullptr)) return fail(c, D2C_EINVAL, "new_k and new_v go together");
    if (!attend && !s.new_k) return fail(c, D2C_EINVAL, "new_k / new_v missing");
    if (s.new_k) {
      if (s.m > s.L) return fail(c, D2C_EINVAL, "more refreshed rows than L");
      if (!aligned(s.new_k, 16) || !aligned(s.new_v, 16) || !aligned(s.idx, 4))
        return fail(c, D2C_EINVAL, "new_k / new_v must be aligned to 16 bytes");
      add(c, s.idx, (size_t)s.m * 4, kReads);
      add(c, s.new_k, s.m * row_bytes(c, c->dims.n_kv_heads), kReads);
      add(c, s.new_v, s.m * row_bytes(c, c->dims.n_kv_heads), kReads);
    }
    add_cache(c, s.cache, s.L, s.new_k ? kRefreshes : kReadsCache);
    if (attend) {
      if (!s.q || !s.out) return fail(c, D2C_EINVAL, "null q or out");
      if (!aligned(s.q, 16) || !aligned(s.out, 16) || !aligned(s.attn_avg, 4))
        return fail(c, D2C_EINVAL, "q and out must be aligned to 16 bytes");
      rows += s.m;
      if (s.attn_avg) tiles += (int64_t)((s.m + 31) / 32) * q8_blocks(s.L);
      add(c, s.q, s.m * row_bytes(c, c->dims.n_heads), kReads);
      add(c, s.out, s.m * row_bytes(c, c->dims.n_heads), kWrites);
      add(c, s.attn_avg, (size_t)s.m * s.L * 4, kWrites);
    }
  }
  if (rows > c->dims.max_rows) return fail(c, D2C_ESHAPE, "query rows exceed max_rows of the handle");
  // a workgroup of 512 for each of these, and a launch holds fewer than 2^32 threads
  if (tiles >= 1 << 23) return fail(c, D2C_ESHAPE, "the averages of the call have 2^23 or more tiles of 32 rows x 64 keys");
  return check_overlap(c);         // (two sequences must not refresh one cache: their order is not defined)
}
int do_update(d2c_q8* c, const d2c_q8_seq* seqs, int batch, hipStream_t st) {
  Q8Update u[kMaxBatch];
  int n = 0;
  for (int i = 0; i < batch; ++i)
    if (seqs[i].m > 0 && seqs[i].new_k)
      u[n++] = Q8Update{ptr(seqs[i].cache), seqs[i].idx, seqs[i].new_k, seqs[i].new_v, seqs[i].m, seqs[i].L};
  return n ? hip(c, launch_q8_update(c->shape, u, n, st), "update") : D2C_OK;
}

}  // namespace

extern "C" {

int d2c_q8_init(const d2c_q8_dims* dims, d2c_q8** out) {
  if (!dims || !out) return fail(nullptr, D2C_EINVAL, "null argument");
  const d2c_q8_dims& D = *dims;
  if (D.n_heads <= 0 || D.n_kv_heads <= 0 || D.n_heads > 1024) return fail(nullptr, D2C_EINVAL, "n_heads must be in 1 .. 1024");
  if (D.n_heads % D.n_kv_heads) return fail(nullptr, D2C_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if (D.head_dim != 64 && D.head_dim != 128) return fail(nullptr, D2C_ESHAPE, "head_dim must be 64 or 128");
  if (D.dtype != D2C_F32 && D.dtype != D2C_BF16) return fail(nullptr, D2C_EINVAL, "dtype must be D2C_F32 or D2C_BF16");
  if (D.max_seq < 0 || D.max_seq > 1 << 24) return fail(nullptr, D2C_EINVAL, "max_seq must be in 0 .. 2^24");
  if (D.max_rows < 0 || D.max_rows > 1 << 16) return fail(nullptr, D2C_EINVAL, "max_rows must be in 0 .. 2^16");
  if (D.max_batch < 0 || D.max_batch > kMaxBatch) return fail(nullptr, D2C_EINVAL, "max_batch must be in 0 .. 256");
  if (D.max_k < 0 || D.max_k > 1 << 16) return fail(nullptr, D2C_EINVAL, "max_k must be in 0 .. 2^16");
  if (D.max_n < 0 || D.max_n > 1 << 20) return fail(nullptr, D2C_EINVAL, "max_n must be in 0 .. 2^20");
  d2c_q8* c = new (std::nothrow) d2c_q8();
  if (!c) return fail(nullptr, D2C_ENOMEM, "out of host memory");
  c->dims = D;
  c->max_batch = std::max(1, (int)D.max_batch);
  c->shape = Q8Shape{D.n_heads, D.n_kv_heads, D.head_dim, D.dtype};
  if (hipGetDevice(&c->device) != hipSuccess) {
    (void)hipGetLastError();
    delete c;
    return fail(nullptr, D2C_EHIP, "hipGetDevice failed");
  }
  size_t bytes = 256;
  if (D.max_seq > 0 && D.max_rows > 0) bytes = std::max(bytes, q8_attention_bytes(c->shape, D.max_rows, c->max_batch));
  if (D.max_k > 0 && D.max_n > 0 && D.max_rows > 0) bytes = std::max(bytes, q8_linear_bytes(D.max_rows, D.max_k));
  const hipError_t e = hipMalloc(&c->ws, bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete c;
    return fail(nullptr, e == hipErrorOutOfMemory ? D2C_ENOMEM : D2C_EHIP, "workspace: ", hipGetErrorString(e));
  }
  c->ws_bytes = (int64_t)bytes;
  *out = c;
  return D2C_OK;
}

int d2c_q8_destroy(d2c_q8* c) {
  if (!c) return D2C_OK;
  if (c->ws) (void)hipFree(c->ws);
  delete c;
  return D2C_OK;
}

const char* d2c_q8_last_error(const d2c_q8* c) { return c ? c->err : g_err; }

int64_t d2c_q8_workspace_bytes(const d2c_q8* c) { return c ? c->ws_bytes : 0; }

int d2c_q8_cache_size(const d2c_q8* c, int64_t rows, int64_t* code_bytes, int64_t* scale_floats) {
  if (!c || !code_bytes || !scale_floats || rows < 0) return D2C_EINVAL;
  const int64_t blocks = (rows + D2C_Q8_BLOCK - 1) / D2C_Q8_BLOCK;
  *code_bytes = blocks * c->dims.n_kv_heads * D2C_Q8_BLOCK * c->dims.head_dim;
  *scale_floats = blocks * c->dims.n_kv_heads;
  return D2C_OK;
}

int d2c_q8_update(d2c_q8* c, const d2c_q8_seq* seqs, int32_t batch, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc || (rc = check_seqs(c, seqs, batch, false))) return rc;
  return do_update(c, seqs, batch, (hipStream_t)stream);
}

int d2c_q8_attention(d2c_q8* c, const d2c_q8_seq* seqs, int32_t batch, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc || (rc = check_seqs(c, seqs, batch, true))) return rc;
  if ((rc = do_update(c, seqs, batch, (hipStream_t)stream))) return rc;
  Q8Attend a[kMaxBatch];
  int n = 0;
  for (int i = 0; i < batch; ++i)
    if (seqs[i].m > 0) a[n++] = Q8Attend{ptr(seqs[i].cache), seqs[i].q, seqs[i].out, seqs[i].attn_avg, seqs[i].m, seqs[i].L};
  return n ? hip(c, launch_q8_attention(c->shape, a, n, c->dims.max_rows, c->max_batch, c->ws, (hipStream_t)stream), "attention") : D2C_OK;
}

int d2c_q8_read(d2c_q8* c, const d2c_q8_cache* cache, int32_t L, const int32_t* idx, int32_t n, void* out_k, void* out_v, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  if (!cache) return fail(c, D2C_EINVAL, "null cache");
  if ((rc = check_cache(c, *cache, L))) return rc;
  if (n < 0 || (!idx && n > L)) return fail(c, D2C_EINVAL, "n outside [0, L]");
  if (n > 1 << 24) return fail(c, D2C_ESHAPE, "more than 2^24 rows");
  if (!aligned(out_k, 16) || !aligned(out_v, 16) || !aligned(idx, 4)) return fail(c, D2C_EINVAL, "outputs must be aligned to 16 bytes");
  if (n == 0 || (!out_k && !out_v)) return D2C_OK;
  c->n_ranges = 0;
  add_cache(c, *cache, L, kReads);
  add(c, idx, (size_t)n * 4, kReads);
  add(c, out_k, n * row_bytes(c, c->dims.n_kv_heads), kWrites);
  add(c, out_v, n * row_bytes(c, c->dims.n_kv_heads), kWrites);
  if ((rc = check_overlap(c))) return rc;
  return hip(c, launch_q8_read(c->shape, ptr(*cache), L, idx, n, out_k, out_v, (hipStream_t)stream), "read");
}

int64_t d2c_q8_weight_bytes(int32_t N, int32_t K) {
  return N <= 0 || K <= 0 ? 0 : ((int64_t)N + 15) / 16 * 16 * (((int64_t)K + 63) / 64 * 64);
}

static int check_linear(d2c_q8* c, int m, int N, int K) {
  if (m < 0 || N <= 0 || K <= 0) return fail(c, D2C_EINVAL, "bad m, N or K");
  if (N > 1 << 20 || K > 1 << 16) return fail(c, D2C_ESHAPE, "N or K too large");
  if (K % (c->dims.dtype == D2C_BF16 ? 8 : 4)) return fail(c, D2C_ESHAPE, "K must be a multiple of 16 bytes of T");
  return D2C_OK;
}

int d2c_q8_plan_linear(int32_t m, int32_t N, int32_t K, int32_t shape[5]) {
  if (!shape || m <= 0 || m > 1 << 16 || N <= 0 || N > 1 << 20 || K <= 0 || K > 1 << 16) return D2C_EINVAL;
  const Q8LinearPlan p = q8_plan_linear(m, N, K);
  shape[0] = p.kernel;
  shape[1] = p.mt;
  shape[2] = p.nt;
  shape[3] = p.waves;
  shape[4] = p.splits;
  return D2C_OK;
}

int d2c_q8_pack(d2c_q8* c, const void* w, int32_t N, int32_t K, int8_t* codes, float* scale, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc || (rc = check_linear(c, 0, N, K))) return rc;
  if (!w || !codes || !scale) return fail(c, D2C_EINVAL, "null buffer");
  if (!aligned(w, 16) || !aligned(codes, 16) || !aligned(scale, 4)) return fail(c, D2C_EINVAL, "w and codes must be aligned to 16 bytes");
  c->n_ranges = 0;
  add(c, w, (size_t)N * K * (c->dims.dtype == D2C_BF16 ? 2 : 4), kReads);
  add(c, codes, (size_t)d2c_q8_weight_bytes(N, K), kWrites);
  add(c, scale, (size_t)N * 4, kWrites);
  if ((rc = check_overlap(c))) return rc;
  return hip(c, launch_q8_pack(c->dims.dtype, w, N, K, codes, scale, (hipStream_t)stream), "pack");
}

int d2c_q8_linear(d2c_q8* c, const void* a, int32_t m, const int8_t* codes, const float* scale, int32_t N, int32_t K, float* out,
                  void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc || (rc = check_linear(c, m, N, K))) return rc;
  if (m > c->dims.max_rows || N > c->dims.max_n || K > c->dims.max_k) return fail(c, D2C_ESHAPE, "m, N or K exceeds max_rows, max_n or max_k");
  if (m == 0) return D2C_OK;
  if (!a || !codes || !scale || !out) return fail(c, D2C_EINVAL, "null buffer");
  if (!aligned(a, 16) || !aligned(codes, 16) || !aligned(scale, 4) || !aligned(out, 4))
    return fail(c, D2C_EINVAL, "a and codes must be aligned to 16 bytes, out to 4");
  c->n_ranges = 0;
  add(c, a, (size_t)m * K * (c->dims.dtype == D2C_BF16 ? 2 : 4), kReads);
  add(c, codes, (size_t)d2c_q8_weight_bytes(N, K), kReads);
  add(c, scale, (size_t)N * 4, kReads);
  add(c, out, (size_t)m * N * 4, kWrites);
  if ((rc = check_overlap(c))) return rc;
  return hip(c, launch_q8_linear(c->dims.dtype, a, m, codes, scale, N, K, out, c->ws, (hipStream_t)stream), "linear");
}

int d2c_q8_weigh(d2c_q8* c, const float* avg, int32_t m, int32_t L, int64_t* weight, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  if (m < 0 || L <= 0) return fail(c, D2C_EINVAL, "bad m or L");
  if (m > 1 << 24 || L > 1 << 24) return fail(c, D2C_ESHAPE, "m or L above 2^24");
  if (m == 0) return D2C_OK;
  if (!avg || !weight) return fail(c, D2C_EINVAL, "null buffer");
  if (!aligned(avg, 4) || !aligned(weight, 8)) return fail(c, D2C_EINVAL, "attn_avg or weight not aligned");
  c->n_ranges = 0;
  add(c, avg, (size_t)m * L * 4, kReads);
  add(c, weight, (size_t)L * 8, kWrites);
  if ((rc = check_overlap(c))) return rc;
  return hip(c, launch_q8_weigh(avg, m, L, weight, (hipStream_t)stream), "weigh");
}

int d2c_q8_evict(d2c_q8* c, const d2c_q8_cache* src, int32_t L, const int64_t* weight, const uint8_t* protect, int32_t n_keep,
                 const d2c_q8_cache* dst, int32_t* kept, int64_t* kept_weight, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  if (!src || !dst) return fail(c, D2C_EINVAL, "null cache");
  if ((rc = check_cache(c, *src, L))) return rc;
  if (n_keep < 0 || n_keep > L) return fail(c, D2C_EINVAL, "n_keep outside [0, L]");
  if (n_keep == 0) return D2C_OK;
  if ((rc = check_cache(c, *dst, n_keep))) return rc;
  if (!weight || !kept) return fail(c, D2C_EINVAL, "null buffer");
  if (!aligned(weight, 8) || !aligned(kept, 4) || !aligned(kept_weight, 8)) return fail(c, D2C_EINVAL, "weight or kept not aligned");
  c->n_ranges = 0;
  add_cache(c, *src, L, kReads);
  add(c, weight, (size_t)L * 8, kReads);
  add(c, protect, (size_t)L, kReads);
  add_cache(c, *dst, n_keep, kWrites);
  add(c, kept, (size_t)n_keep * 4, kWrites);
  add(c, kept_weight, (size_t)n_keep * 8, kWrites);
  if ((rc = check_overlap(c))) return rc;
  hipStream_t st = (hipStream_t)stream;
  if ((rc = hip(c, launch_q8_keep(weight, protect, L, n_keep, kept, kept_weight, st), "evict"))) return rc;
  return hip(c, launch_q8_compact(c->shape, ptr(*src), kept, n_keep, ptr(*dst), st), "evict");
}

}  // extern "C"
