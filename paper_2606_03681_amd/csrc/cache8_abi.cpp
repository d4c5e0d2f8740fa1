// Host side of the C ABI declared in include/tfm_cache.h: argument validation and launches.
#include "tfm_cache.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "cache8.h"
#include "ends.h"
#include "prof.h"

namespace {

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return tfm::abi_fail(code, buf);
}

constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr double kMaxReach = 281474976710656.0;  // 2^48 elements from the first row to the last
constexpr int64_t kMax31 = 0x7fffffff;
bool aligned(const void* p, size_t a) { return p && ((uintptr_t)p % a) == 0; }
bool aligned_or_null(const void* p, size_t a) { return !p || ((uintptr_t)p % a) == 0; }
size_t elem(int32_t d) { return d == TFM_BF16 ? 2 : 4; }

#define HIPCHK(...)                                                                     \
  do {                                                                                  \
    hipError_t e_ = (__VA_ARGS__);                                                      \
    if (e_ != hipSuccess)                                                               \
      return fail(TFM_ERR_HIP, "%s failed: %s", #__VA_ARGS__, hipGetErrorString(e_));   \
  } while (0)

#define STEP(name, ...)              \
  do {                               \
    tfm::prof_begin(name, st);       \
    HIPCHK(__VA_ARGS__);             \
    tfm::prof_end(st);               \
  } while (0)

size_t pool_size(const tfm_cache8* c) {
  return tfm::cache8_pool_bytes(c->heads, c->d, c->page, c->n_pages);
}

int pool_check(const tfm_cache8* c) {
  if (!c) return fail(TFM_ERR_POINTER, "the cache's description is null");
  if (c->heads < 1 || c->heads > 4096) return fail(TFM_ERR_DIMS, "heads=%d outside [1, 4096]", c->heads);
  if (c->d != 16 && c->d != 32 && c->d != 64 && c->d != 128)
    return fail(TFM_ERR_HEAD_DIM, "d=%d is not 16, 32, 64 or 128", c->d);
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256)
    return fail(TFM_ERR_DIMS, "page=%d is not 16, 32, 64, 128 or 256", c->page);
  if (c->n_pages < 1) return fail(TFM_ERR_DIMS, "n_pages=%d must be >= 1", c->n_pages);
  if ((double)c->n_pages * c->heads * c->page * c->d > 35184372088832.0)
    return fail(TFM_ERR_DIMS, "the pool has more than 2^46 bytes");
  return TFM_OK;
}

int batch_check(const tfm_cache8* c, int32_t B, int32_t L, int32_t max_pages, int32_t dtype) {
  if (B < 0 || L < 0) return fail(TFM_ERR_DIMS, "B=%d or L=%d is negative", B, L);
  if (max_pages < 0 || (int64_t)max_pages * c->page > (1 << 30))
    return fail(TFM_ERR_DIMS, "max_pages=%d of %d rows outside [0, 2^30]", max_pages, c->page);
  if ((int64_t)B * max_pages > kMax31)
    return fail(TFM_ERR_DIMS, "%d x %d page indices are more than 2^31 - 1", B, max_pages);
  if (dtype != TFM_F32 && dtype != TFM_BF16)
    return fail(TFM_ERR_DIMS, "dtype=%d is not a tfm_dtype", dtype);
  return TFM_OK;
}

// Rows (sequence, row, head) of d elements; apart: none may overlap another.
int strides_check(const char* name, const int64_t* stride, const int32_t* n, int d, bool apart) {
  double reach = d;
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i)
    if (stride[i] < 0 || stride[i] > kMaxStride)
      return fail(TFM_ERR_DIMS, "%s[%d]=%lld outside [0, 2^40]", name, i, (long long)stride[i]);
  std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  for (int i : order) {
    if (n[i] <= 1) continue;
    if (apart && (double)stride[i] < reach)
      return fail(TFM_ERR_DIMS, "rows overlap: %s[%d]=%lld is less than the %.0f elements that the "
                                "inner axes reach", name, i, (long long)stride[i], reach);
    reach += (double)(n[i] - 1) * (double)stride[i];
  }
  if (reach > kMaxReach)
    return fail(TFM_ERR_DIMS, "%s: the rows reach over more than 2^48 elements", name);
  return TFM_OK;
}

// Elements from the first row's start to the last row's.
double reach_of(const int64_t* stride, int32_t a, int32_t b, int32_t c) {
  return (double)(a - 1) * (double)stride[0] + (double)(b - 1) * (double)stride[1] +
         (double)(c - 1) * (double)stride[2];
}
tfm::Cache8Geo geo_of(const tfm_cache8* c, void* pool, int32_t max_pages, const int32_t* pages) {
  return tfm::cache8_geo(c->heads, c->d, c->page, c->n_pages, pool, max_pages, pages);
}

int pool_given(const tfm_cache8* c, const void* pool, size_t bytes) {
  if (!aligned(pool, 16)) return fail(TFM_ERR_POINTER, "pool null or not 16-byte aligned");
  if (bytes < pool_size(c))
    return fail(TFM_ERR_BUFFER, "pool has %zu bytes, %zu required", bytes, pool_size(c));
  return TFM_OK;
}

int rows_check(const tfm_cache8* c, const tfm_cache8_rows* r) {
  int rc = pool_check(c);
  if (rc) return rc;
  if (!r) return fail(TFM_ERR_POINTER, "the rows' description is null");
  rc = batch_check(c, r->B, r->L, r->max_pages, r->dtype);
  if (rc) return rc;
  const int32_t n[3] = {r->B, r->L, c->heads};
  rc = strides_check("stride_k", r->stride_k, n, c->d, false);
  return rc ? rc : strides_check("stride_v", r->stride_v, n, c->d, false);
}

int query_check(const tfm_cache8* c, const tfm_cache8_query* a, tfm::Cache8Attend& t) {
  int rc = pool_check(c);
  if (rc) return rc;
  if (!a) return fail(TFM_ERR_POINTER, "the query's description is null");
  rc = batch_check(c, a->B, a->L, a->max_pages, a->dtype);
  if (rc) return rc;
  if (a->heads < 1 || a->heads > (1 << 16) || a->heads % c->heads)
    return fail(TFM_ERR_DIMS, "heads=%d is not a multiple of the cache's %d in [1, 2^16]", a->heads,
                c->heads);
  if ((double)a->B * a->L * a->heads > (double)kMax31)
    return fail(TFM_ERR_DIMS, "%d x %d x %d query rows are more than 2^31 - 1", a->B, a->L, a->heads);
  if ((int64_t)a->L * a->heads > (1 << 26))
    return fail(TFM_ERR_DIMS, "%d rows of %d heads are more than 2^26", a->L, a->heads);
  if (a->max_len < 0) return fail(TFM_ERR_DIMS, "max_len=%d is negative", a->max_len);
  if (!(std::fabs(a->scale) <= 0x1p64f))  // (times log2 e and a power of at most 2^48: a float32)
    return fail(TFM_ERR_DIMS, "scale=%g outside [-2^64, 2^64]", (double)a->scale);
  const int32_t n[3] = {a->B, a->L, a->heads};
  rc = strides_check("stride_q", a->stride_q, n, c->d, false);
  if (rc) return rc;
  rc = strides_check("stride_out", a->stride_out, n, c->d, true);
  if (rc) return rc;
  t = tfm::Cache8Attend{};
  t.g = geo_of(c, nullptr, a->max_pages, nullptr);
  t.B = a->B; t.L = a->L; t.heads = a->heads; t.causal = a->causal != 0;
  const int64_t room = (int64_t)a->max_pages * c->page;
  t.max_rows = (int32_t)(a->max_len > 0 && a->max_len < room ? a->max_len : room);
  t.plan_B = t.B;
  t.scale_log2 = (float)(a->scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) t.sq[i] = a->stride_q[i], t.so[i] = a->stride_out[i];
  return TFM_OK;
}

}  // namespace

extern "C" {

size_t tfm_cache8_bytes(const tfm_cache8* c) { return pool_check(c) ? 0 : pool_size(c); }

int tfm_cache8_append(const tfm_cache8* c, const tfm_cache8_rows* r, const void* k, const void* v,
                      const int32_t* pages, const int32_t* lens, const int32_t* n_new, void* pool,
                      size_t pool_bytes, void* stream) {
  int rc = rows_check(c, r);
  if (rc) return rc;
  rc = pool_given(c, pool, pool_bytes);
  if (rc) return rc;
  if (r->B == 0 || r->L == 0 || r->max_pages == 0) return TFM_OK;
  const size_t es = elem(r->dtype);
  if (!aligned(k, es) || !aligned(v, es))
    return fail(TFM_ERR_POINTER, "k and v must be non-null and aligned to their elements");
  if (!aligned_or_null(pages, 4) || !aligned_or_null(lens, 4) || !aligned_or_null(n_new, 4))
    return fail(TFM_ERR_POINTER, "pages, lens and n_new must be 4-byte aligned");
  if (tfm::overlap(k, (reach_of(r->stride_k, r->B, r->L, c->heads) + c->d) * es, pool, (double)pool_size(c)) ||
      tfm::overlap(v, (reach_of(r->stride_v, r->B, r->L, c->heads) + c->d) * es, pool, (double)pool_size(c)))
    return fail(TFM_ERR_POINTER, "k or v overlaps the pool");
  hipStream_t st = (hipStream_t)stream;
  tfm::Cache8Append a;
  a.g = geo_of(c, pool, r->max_pages, pages);
  a.B = r->B; a.L = r->L;
  for (int i = 0; i < 3; ++i) a.sk[i] = r->stride_k[i], a.sv[i] = r->stride_v[i];
  a.lens = lens; a.n_new = n_new;
  if (r->dtype == TFM_BF16)
    STEP("cache8_append/hbm", tfm::launch_cache8_append(a, (const tfm::bf16*)k, (const tfm::bf16*)v, st));
  else
    STEP("cache8_append/hbm", tfm::launch_cache8_append(a, (const float*)k, (const float*)v, st));
  return TFM_OK;
}

size_t tfm_cache8_attend_workspace_bytes(const tfm_cache8* c, const tfm_cache8_query* a) {
  tfm::Cache8Attend t;
  if (query_check(c, a, t)) return 0;
  return tfm::cache8_attend_bytes(t, a->dtype == TFM_F32);
}

int tfm_cache8_attend(const tfm_cache8* c, const tfm_cache8_query* a, const void* q,
                      const int32_t* pages, const int32_t* lens, const int32_t* n_rows,
                      const void* pool, size_t pool_bytes, void* out, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream) {
  tfm::Cache8Attend t;
  int rc = query_check(c, a, t);
  if (rc) return rc;
  rc = pool_given(c, pool, pool_bytes);
  if (rc) return rc;
  if (a->B == 0 || a->L == 0) return TFM_OK;
  const size_t es = elem(a->dtype);
  if (!aligned(q, es) || !aligned(out, es) || !aligned(lens, 4))
    return fail(TFM_ERR_POINTER, "q, out and lens must be non-null and aligned to their elements");
  if (!aligned_or_null(pages, 4) || !aligned_or_null(n_rows, 4) || !aligned_or_null(lse, 4))
    return fail(TFM_ERR_POINTER, "pages, n_rows and lse must be 4-byte aligned");
  const double span = (reach_of(a->stride_out, a->B, a->L, a->heads) + c->d) * es;
  if (q == out && !std::equal(a->stride_q, a->stride_q + 3, a->stride_out))
    return fail(TFM_ERR_POINTER, "out is q, with other strides");
  if (tfm::overlap(out, span, pool, (double)pool_size(c)) ||
      tfm::overlap(out, span, lse, 4.0 * a->B * a->L * a->heads) ||
      tfm::overlap(lse, 4.0 * a->B * a->L * a->heads, pool, (double)pool_size(c)))
    return fail(TFM_ERR_POINTER, "one of out, the pool and lse overlaps another");
  const size_t need = tfm::cache8_attend_bytes(t, a->dtype == TFM_F32);
  if (need && !aligned(workspace, 16))
    return fail(TFM_ERR_POINTER, "workspace null or not 16-byte aligned");
  if (workspace_bytes < need)
    return fail(TFM_ERR_BUFFER, "workspace has %zu bytes, %zu required", workspace_bytes, need);
  hipStream_t st = (hipStream_t)stream;
  t.g = geo_of(c, const_cast<void*>(pool), a->max_pages, pages);
  t.lens = lens; t.n_rows = n_rows; t.lse = lse; t.ws = workspace;
  if (a->dtype == TFM_BF16)
    STEP("cache8_attend/mfma", tfm::launch_cache8_attend(t, (const tfm::bf16*)q, (tfm::bf16*)out, st));
  else
    STEP("cache8_attend/mfma", tfm::launch_cache8_attend(t, (const float*)q, (float*)out, st));
  return TFM_OK;
}

}  // extern "C"
