// C ABI of the paged cache (see include/d2c_pg.h): argument validation, workspace and the order of kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <new>

#include "../../include/d2c_pg.h"
#include "internal.h"
#include "pg.h"

using namespace d2c;

constexpr int kMaxBuffers = 16;

struct d2c_pg {
  d2c_pg_dims dims{};
  PgShape shape{};
  PgRotation rotation{};
  PgWorkspace sizes{};
  int device = 0, cus = 0, max_batch = 1;
  void* ws = nullptr;            // of d2c_pg_attention: calls do not overlap
  struct Range {
    uintptr_t at, end;
    bool writes;
  } ranges[kMaxBuffers];         // of the call that is checked
  int n_ranges = 0;
  char err[256] = {};
};

namespace {

thread_local char g_err[256] = {};     // of this thread's last d2c_pg_init

int fail(d2c_pg* c, int code, const char* msg, const char* more = "") {
  snprintf(c ? c->err : g_err, 256, "%s%s", msg, more);
  return code;
}
int hip(d2c_pg* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return D2C_OK;
  (void)hipGetLastError();
  snprintf(c->err, sizeof c->err, "%s: %s", what, hipGetErrorString(e));
  return D2C_EHIP;
}
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int size_of(int dtype) { return dtype == D2C_BF16 ? 2 : 4; }

void add(d2c_pg* c, const void* p, size_t bytes, bool writes) {
  if (p && bytes) c->ranges[c->n_ranges++] = d2c_pg::Range{(uintptr_t)p, (uintptr_t)p + bytes, writes};
}
int check_overlap(d2c_pg* c) {
  for (int i = 0; i < c->n_ranges; ++i)
    for (int j = 0; j < i; ++j)
      if ((c->ranges[i].writes || c->ranges[j].writes) && c->ranges[i].at < c->ranges[j].end && c->ranges[j].at < c->ranges[i].end)
        return fail(c, D2C_EINVAL, "a buffer that the call writes overlaps another of its buffers");
  return D2C_OK;
}
int check_device(d2c_pg* c) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(c, D2C_EHIP, "hipGetDevice failed");
  return dev == c->device ? D2C_OK : fail(c, D2C_EINVAL, "another device is current than the handle's");
}
size_t page_bytes(const d2c_pg* c) {
  return (size_t)c->dims.page_rows * c->dims.n_kv_heads * c->dims.head_dim * size_of(c->dims.dtype);
}
int check_cache(d2c_pg* c, const d2c_pg_cache* k, bool writes) {
  if (!k || !k->k || !k->v) return fail(c, D2C_EINVAL, "null cache");
  if (k->n_pages < 1) return fail(c, D2C_EINVAL, "n_pages must be positive");
  if (!aligned(k->k, 16) || !aligned(k->v, 16)) return fail(c, D2C_EINVAL, "pages must be aligned to 16 bytes");
  add(c, k->k, k->n_pages * page_bytes(c), writes);
  add(c, k->v, k->n_pages * page_bytes(c), writes);
  return D2C_OK;
}
// D2C_OK with *none set where there is nothing to do
int check_batch(d2c_pg* c, const d2c_pg_batch* b, bool* none) {
  if (!b) return fail(c, D2C_EINVAL, "null batch");
  if (b->batch < 0 || b->n_rows < 0 || b->page_cols < 0) return fail(c, D2C_EINVAL, "negative batch, n_rows or page_cols");
  if (b->batch > c->max_batch) return fail(c, D2C_ESHAPE, "batch exceeds max_batch of the handle");
  if (b->n_rows > 1 << 24) return fail(c, D2C_ESHAPE, "more than 2^24 rows");
  if ((int64_t)b->page_cols * c->dims.page_rows > 1 << 30) return fail(c, D2C_ESHAPE, "page_cols * page_rows above 2^30");
  *none = b->batch == 0 || b->n_rows == 0;
  if (*none) return D2C_OK;
  if (!b->row_start || !b->length || (!b->pages && b->page_cols > 0)) return fail(c, D2C_EINVAL, "null row_start, length or pages");
  if (!aligned(b->row_start, 4) || !aligned(b->length, 4) || !aligned(b->pages, 4) || !aligned(b->at, 4) || !aligned(b->origin, 4))
    return fail(c, D2C_EINVAL, "an array of the batch is not aligned");
  add(c, b->row_start, ((size_t)b->batch + 1) * 4, false);
  add(c, b->length, (size_t)b->batch * 4, false);
  add(c, b->pages, (size_t)b->batch * b->page_cols * 4, false);
  add(c, b->at, (size_t)b->n_rows * 4, false);
  add(c, b->origin, (size_t)b->batch * 4, false);
  return D2C_OK;
}
PgBatch batch_of(const d2c_pg_batch& b) { return PgBatch{b.row_start, b.length, b.pages, b.at, b.origin, b.batch, b.n_rows, b.page_cols}; }
PgPages pages_of(const d2c_pg_cache& k) { return PgPages{k.k, k.v, k.n_pages}; }

// n rows of `width` values of a type, ld from row to row
int check_rows(d2c_pg* c, const void* p, int64_t n, int64_t width, int64_t ld, int dtype, bool writes) {
  if (!p) return fail(c, D2C_EINVAL, "null rows");
  if (ld < width || ld > (int64_t)1 << 40) return fail(c, D2C_EINVAL, "a row pitch is smaller than the row, or above 2^40");
  if (!aligned(p, 16) || ld * size_of(dtype) % 16) return fail(c, D2C_EINVAL, "rows and their pitch must be multiples of 16 bytes");
  if (n > 0) add(c, p, (size_t)((n - 1) * ld + width) * size_of(dtype), writes);
  return D2C_OK;
}

}  // namespace

extern "C" {

int d2c_pg_init(const d2c_pg_dims* dims, d2c_pg** out) {
  if (!dims || !out) return fail(nullptr, D2C_EINVAL, "null argument");
  const d2c_pg_dims& D = *dims;
  if (D.n_heads <= 0 || D.n_kv_heads <= 0 || D.n_heads > 1024) return fail(nullptr, D2C_EINVAL, "n_heads must be in 1 .. 1024");
  if (D.n_heads % D.n_kv_heads) return fail(nullptr, D2C_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if (D.head_dim != 64 && D.head_dim != 128) return fail(nullptr, D2C_ESHAPE, "head_dim must be 64 or 128");
  if (D.dtype != D2C_F32 && D.dtype != D2C_BF16) return fail(nullptr, D2C_EINVAL, "dtype must be D2C_F32 or D2C_BF16");
  if (D.page_rows != 32 && D.page_rows != 64 && D.page_rows != 128 && D.page_rows != 256)
    return fail(nullptr, D2C_ESHAPE, "page_rows must be 32, 64, 128 or 256");
  if (D.max_rows < 0 || D.max_rows > 1 << 20) return fail(nullptr, D2C_EINVAL, "max_rows must be in 0 .. 2^20");
  if (D.max_batch < 0 || D.max_batch > kPgMaxBatch) return fail(nullptr, D2C_EINVAL, "max_batch must be in 0 .. 1024");
  if (D.n_pairs < 0 || D.n_pairs % 8 || 2 * D.n_pairs > D.head_dim) return fail(nullptr, D2C_EINVAL, "n_pairs must be a multiple of 8 up to head_dim / 2");
  if (D.n_axes < 0 || D.n_axes > 4) return fail(nullptr, D2C_EINVAL, "n_axes must be in 0 .. 4");
  if (D.pairing != D2C_PG_HALVES && D.pairing != D2C_PG_NEIGHBOURS) return fail(nullptr, D2C_EINVAL, "pairing must be D2C_PG_HALVES or D2C_PG_NEIGHBOURS");
  const int axes = std::max(1, (int)D.n_axes);
  for (int i = 0; i < D.n_pairs; ++i) {
    if (!(std::fabs(D.freq[i]) <= 65536.0)) return fail(nullptr, D2C_EINVAL, "a frequency is not finite or above 2^16");
    if (D.axis[i] >= axes) return fail(nullptr, D2C_EINVAL, "a pair's axis is not below n_axes");
  }
  d2c_pg* c = new (std::nothrow) d2c_pg();
  if (!c) return fail(nullptr, D2C_ENOMEM, "out of host memory");
  c->dims = D;
  c->max_batch = std::max(1, (int)D.max_batch);
  c->shape = PgShape{D.n_heads, D.n_kv_heads, D.head_dim, D.dtype, D.page_rows == 32 ? 5 : D.page_rows == 64 ? 6 : D.page_rows == 128 ? 7 : 8};
  for (int i = 0; i < D.n_pairs; ++i) {
    c->rotation.turns[i] = D.freq[i] / 6.283185307179586476925;
    c->rotation.axis[i] = D.axis[i];
  }
  c->rotation.n_pairs = D.n_pairs;
  c->rotation.n_axes = axes;
  c->rotation.pairing = D.pairing;
  c->sizes = pg_workspace(c->shape, D.max_rows, c->max_batch);
  if (hipGetDevice(&c->device) != hipSuccess || hipDeviceGetAttribute(&c->cus, hipDeviceAttributeMultiprocessorCount, c->device) != hipSuccess) {
    (void)hipGetLastError();
    delete c;
    return fail(nullptr, D2C_EHIP, "no device");
  }
  if (c->sizes.bytes > 0) {
    const hipError_t e = hipMalloc(&c->ws, c->sizes.bytes);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return fail(nullptr, e == hipErrorOutOfMemory ? D2C_ENOMEM : D2C_EHIP, "workspace: ", hipGetErrorString(e));
    }
  }
  *out = c;
  return D2C_OK;
}

int d2c_pg_destroy(d2c_pg* c) {
  if (!c) return D2C_OK;
  if (c->ws) (void)hipFree(c->ws);
  delete c;
  return D2C_OK;
}

const char* d2c_pg_last_error(const d2c_pg* c) { return c ? c->err : g_err; }

int64_t d2c_pg_workspace_bytes(const d2c_pg* c) { return c ? (int64_t)c->sizes.bytes : 0; }

int d2c_pg_cache_size(const d2c_pg* c, int64_t n_pages, int64_t* bytes) {
  if (!c || !bytes || n_pages < 0 || n_pages > 0x7fffffff) return D2C_EINVAL;
  *bytes = n_pages * (int64_t)page_bytes(c);
  return D2C_OK;
}

int d2c_pg_rotate(d2c_pg* c, const void* x, int64_t x_ld, int32_t x_dtype, int32_t n, int32_t heads, const int32_t* pos, int32_t inverse, void* out,
                  int64_t out_ld, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  if (c->dims.n_pairs == 0) return fail(c, D2C_EINVAL, "the handle was made without a rotation");
  if (n < 0 || heads <= 0 || heads > 1024) return fail(c, D2C_EINVAL, "bad n or heads");
  if (n > 1 << 24) return fail(c, D2C_ESHAPE, "more than 2^24 rows");
  if (x_dtype != D2C_F32 && x_dtype != c->dims.dtype) return fail(c, D2C_EINVAL, "x_dtype must be D2C_F32 or the handle's");
  if (n == 0) return D2C_OK;
  c->n_ranges = 0;
  const int64_t width = (int64_t)heads * c->dims.head_dim;
  const bool in_place = x == out && x_ld == out_ld && x_dtype == c->dims.dtype;      // each thread writes only what it has read itself
  if ((rc = check_rows(c, x, n, width, x_ld, x_dtype, false))) return rc;
  if (in_place) c->n_ranges = 0;
  if ((rc = check_rows(c, out, n, width, out_ld, c->dims.dtype, true))) return rc;
  if (!pos || !aligned(pos, 4)) return fail(c, D2C_EINVAL, "pos is null or not aligned");
  add(c, pos, (size_t)c->rotation.n_axes * n * 4, false);
  if ((rc = check_overlap(c))) return rc;
  PgRows r{};
  r.q = x;
  r.q_ld = x_ld;
  r.q_out = out;
  r.q_out_ld = out_ld;
  r.pos = pos;
  r.src_dtype = x_dtype;
  r.q_heads = heads;
  r.sign = inverse ? -1.f : 1.f;
  return hip(c, launch_pg_rows(c->shape, c->rotation, PgPages{}, nullptr, n, r, (hipStream_t)stream), "rotate");
}

int d2c_pg_append(d2c_pg* c, const d2c_pg_cache* cache, const d2c_pg_batch* batch, const d2c_pg_new* rows, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  bool none = false;
  c->n_ranges = 0;
  if ((rc = check_cache(c, cache, true)) || (rc = check_batch(c, batch, &none))) return rc;
  if (!rows) return fail(c, D2C_EINVAL, "null rows");
  if (rows->dtype != D2C_F32 && rows->dtype != c->dims.dtype) return fail(c, D2C_EINVAL, "dtype must be D2C_F32 or the handle's");
  if ((rows->q == nullptr) != (rows->q_out == nullptr)) return fail(c, D2C_EINVAL, "q and q_out go together");
  if (none) return D2C_OK;
  const int64_t n = batch->n_rows, d_q = (int64_t)c->dims.n_heads * c->dims.head_dim, d_kv = (int64_t)c->dims.n_kv_heads * c->dims.head_dim;
  if ((rc = check_rows(c, rows->k, n, d_kv, rows->k_ld, rows->dtype, false))) return rc;
  if ((rc = check_rows(c, rows->v, n, d_kv, rows->v_ld, rows->dtype, false))) return rc;
  if (rows->q) {
    if ((rc = check_rows(c, rows->q, n, d_q, rows->q_ld, rows->dtype, false))) return rc;
    if ((rc = check_rows(c, rows->q_out, n, d_q, rows->q_out_ld, c->dims.dtype, true))) return rc;
  }
  if (!aligned(rows->pos, 4)) return fail(c, D2C_EINVAL, "pos is not aligned");
  if (c->dims.n_pairs > 0) add(c, rows->pos, (size_t)c->rotation.n_axes * n * 4, false);
  if ((rc = check_overlap(c))) return rc;
  PgRows r{};
  r.q = rows->q;
  r.k = rows->k;
  r.v = rows->v;
  r.q_ld = rows->q_ld;
  r.k_ld = rows->k_ld;
  r.v_ld = rows->v_ld;
  r.q_out = rows->q_out;
  r.q_out_ld = rows->q_out_ld;
  r.pos = rows->pos;
  r.src_dtype = rows->dtype;
  r.q_heads = c->dims.n_heads;
  r.sign = 1.f;
  const PgBatch b = batch_of(*batch);
  return hip(c, launch_pg_rows(c->shape, c->rotation, pages_of(*cache), &b, (int)n, r, (hipStream_t)stream), "append");
}

int d2c_pg_read(d2c_pg* c, const d2c_pg_cache* cache, const d2c_pg_batch* batch, void* out_k, int64_t k_ld, void* out_v, int64_t v_ld, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  bool none = false;
  c->n_ranges = 0;
  if ((rc = check_cache(c, cache, false)) || (rc = check_batch(c, batch, &none))) return rc;
  if (none || (!out_k && !out_v)) return D2C_OK;
  const int64_t d_kv = (int64_t)c->dims.n_kv_heads * c->dims.head_dim;
  if (out_k && (rc = check_rows(c, out_k, batch->n_rows, d_kv, k_ld, c->dims.dtype, true))) return rc;
  if (out_v && (rc = check_rows(c, out_v, batch->n_rows, d_kv, v_ld, c->dims.dtype, true))) return rc;
  if ((rc = check_overlap(c))) return rc;
  return hip(c, launch_pg_read(c->shape, pages_of(*cache), batch_of(*batch), out_k, k_ld, out_v, v_ld, (hipStream_t)stream), "read");
}

int d2c_pg_attention(d2c_pg* c, const d2c_pg_cache* cache, const d2c_pg_batch* batch, const d2c_pg_attend* args, void* stream) {
  if (!c) return D2C_EINVAL;
  int rc = check_device(c);
  if (rc) return rc;
  bool none = false;
  c->n_ranges = 0;
  if ((rc = check_cache(c, cache, false)) || (rc = check_batch(c, batch, &none))) return rc;
  if (!args) return fail(c, D2C_EINVAL, "null args");
  if (batch->n_rows > c->dims.max_rows) return fail(c, D2C_ESHAPE, "n_rows exceeds max_rows of the handle");
  if (args->block < 0 || args->window < 0 || args->block > 1 << 30 || args->window > 1 << 30) return fail(c, D2C_EINVAL, "block and window must be in 0 .. 2^30");
  // (above it the product with log2(e) is no float, and a score of 0 times that no number)
  if (!(args->scale >= 0.f) || !(args->scale <= 0x1p127f)) return fail(c, D2C_EINVAL, "scale must be positive and at most 2^127, or 0");
  if (none) return D2C_OK;
  const int64_t n = batch->n_rows, d_q = (int64_t)c->dims.n_heads * c->dims.head_dim;
  if ((rc = check_rows(c, args->q, n, d_q, args->q_ld, c->dims.dtype, false))) return rc;
  if ((rc = check_rows(c, args->out, n, d_q, args->out_ld, c->dims.dtype, true))) return rc;
  if (args->attn_avg) {
    if (args->avg_ld < 1 || args->avg_ld > 1 << 30) return fail(c, D2C_EINVAL, "avg_ld must be in 1 .. 2^30");
    if (!aligned(args->attn_avg, 4)) return fail(c, D2C_EINVAL, "attn_avg is not aligned");
    add(c, args->attn_avg, (size_t)n * args->avg_ld * 4, true);
  }
  if ((rc = check_overlap(c))) return rc;
  PgAttend a{args->q, args->out, args->attn_avg, args->q_ld, args->out_ld, args->avg_ld, args->block, args->window,
             args->scale > 0.f ? args->scale : 1.f / std::sqrt((float)c->dims.head_dim)};
  return hip(c, launch_pg_attention(c->shape, pages_of(*cache), batch_of(*batch), a, c->sizes, c->ws, c->cus, (hipStream_t)stream), "attention");
}

}  // extern "C"
