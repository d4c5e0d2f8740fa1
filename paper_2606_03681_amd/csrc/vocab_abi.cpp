// Host side of the C ABI declared in include/tfm_vocab.h: argument validation, workspace layouts
// and launch sequences of the embedding, the distillation loss and the sampler.
#include "tfm_vocab.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "ends.h"
#include "prof.h"
#include "vocab.h"

namespace {

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return tfm::abi_fail(code, buf);
}

constexpr int64_t kMaxRows = int64_t(1) << 27;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr double kMaxReach = 281474976710656.0;  // 2^48 elements from the first row to the last
bool aligned(const void* p, size_t a) { return p && ((uintptr_t)p % a) == 0; }
bool aligned_or_null(const void* p, size_t a) { return !p || ((uintptr_t)p % a) == 0; }
bool is_dtype(int32_t d) { return d == TFM_F32 || d == TFM_BF16; }
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

// ---- embedding ------------------------------------------------------------------------------

int embed_check(const tfm_embed* e, tfm::EmbedGeo& g) {
  if (!e) return fail(TFM_ERR_POINTER, "the embedding's description is null");
  double rows = 1.0, reach = 0.0;
  for (int i = 0; i < 3; ++i) {
    if (e->n[i] < 0) return fail(TFM_ERR_DIMS, "n[%d]=%d is negative", i, e->n[i]);
    if (e->stride[i] < 0 || e->stride[i] > kMaxStride)
      return fail(TFM_ERR_DIMS, "stride[%d]=%lld outside [0, 2^40]", i, (long long)e->stride[i]);
    rows *= e->n[i];
    if (e->n[i] > 1) reach += (double)(e->n[i] - 1) * (double)e->stride[i];
  }
  if (reach > kMaxReach) return fail(TFM_ERR_DIMS, "the rows reach over more than 2^48 elements");
  if (rows > (double)kMaxRows)
    return fail(TFM_ERR_DIMS, "%d x %d x %d ids are more than 2^27", e->n[0], e->n[1], e->n[2]);
  if (e->V < 1 || e->V > (1 << 24)) return fail(TFM_ERR_DIMS, "V=%d outside [1, 2^24]", e->V);
  if (e->E < 1 || e->E > (1 << 16)) return fail(TFM_ERR_DIMS, "E=%d outside [1, 2^16]", e->E);
  if (!is_dtype(e->dtype) || !is_dtype(e->table_dtype))
    return fail(TFM_ERR_DIMS, "dtype=%d or table_dtype=%d is not a tfm_dtype", e->dtype,
                e->table_dtype);
  if (!std::isfinite(e->scale)) return fail(TFM_ERR_DIMS, "scale is not finite");
  g.N = (int64_t)rows;
  for (int i = 0; i < 3; ++i) g.stride[i] = e->stride[i];
  g.n1 = e->n[1]; g.n2 = e->n[2];
  g.m1 = g.n1 > 1 ? ~uint64_t(0) / (uint64_t)g.n1 + 1 : 0;
  g.m2 = g.n2 > 1 ? ~uint64_t(0) / (uint64_t)g.n2 + 1 : 0;
  g.E = e->E; g.V = e->V;
  g.scale = e->scale;
  return TFM_OK;
}

// Rows apart: by falling stride each longer axis steps past everything the inner ones reach.
int rows_apart(const tfm_embed* e) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return e->stride[a] < e->stride[b]; });
  double reach = e->E;  // elements from a row's start that the axes so far cover
  for (int i : order) {
    if (e->n[i] <= 1) continue;
    if ((double)e->stride[i] < reach)
      return fail(TFM_ERR_DIMS, "rows overlap: stride[%d]=%lld is less than the %.0f elements that "
                                "the inner axes reach", i, (long long)e->stride[i], reach);
    reach += (double)(e->n[i] - 1) * (double)e->stride[i];
  }
  return TFM_OK;
}

// ---- distillation ----------------------------------------------------------------------------

struct DistillWs {
  size_t wsum, lsum, row_loss, split, total;
};
DistillWs distill_ws(const tfm_distill* d) {
  DistillWs w;
  w.wsum = 0;
  w.lsum = w.wsum + sizeof(double) * tfm::DISTILL_WPARTS;
  w.row_loss = w.lsum + sizeof(double) * tfm::DISTILL_WPARTS;
  w.split = w.row_loss + ((size_t)d->N * 4 + 255) / 256 * 256;
  w.total = w.split + tfm::distill_split_bytes(d->N, d->V, d->k);
  return w;
}

int logits_check(int32_t N, int32_t V, int32_t dtype, int64_t ld) {
  if (N < 0 || N > kMaxRows) return fail(TFM_ERR_DIMS, "N=%d outside [0, 2^27]", N);
  if (V < 1 || V > tfm::VOCAB_VMAX) return fail(TFM_ERR_DIMS, "V=%d outside [1, 2^18]", V);
  if (ld < V || ld > kMaxStride)
    return fail(TFM_ERR_DIMS, "ld=%lld outside [V=%d, 2^40]", (long long)ld, V);
  if (N > 1 && (double)(N - 1) * (double)ld > kMaxReach)
    return fail(TFM_ERR_DIMS, "the rows reach over more than 2^48 elements");
  if (!is_dtype(dtype)) return fail(TFM_ERR_DIMS, "dtype=%d is not a tfm_dtype", dtype);
  return TFM_OK;
}

int distill_check(const tfm_distill* d) {
  if (!d) return fail(TFM_ERR_POINTER, "the distillation's description is null");
  int rc = logits_check(d->N, d->V, d->dtype, d->ld);
  if (rc) return rc;
  if (d->k < 1 || d->k > tfm::DISTILL_KMAX)
    return fail(TFM_ERR_DIMS, "k=%d outside [1, %d]", d->k, tfm::DISTILL_KMAX);
  if (d->tail != 0 && d->tail != 1) return fail(TFM_ERR_DIMS, "tail=%d is not 0 or 1", d->tail);
  if (!(d->temperature >= 0x1p-20f && d->temperature <= 0x1p20f))
    return fail(TFM_ERR_DIMS, "temperature outside [2^-20, 2^20]");
  if (!(d->alpha >= 0.f && d->alpha <= 1.f))
    return fail(TFM_ERR_DIMS, "alpha must lie in [0, 1]");
  return TFM_OK;
}

}  // namespace

extern "C" {

size_t tfm_embed_workspace_bytes(const tfm_embed* e) {
  tfm::EmbedGeo g;
  if (embed_check(e, g)) return 0;
  return tfm::embed_bwd_bytes(g);
}

int tfm_embed_fwd(const tfm_embed* e, const int32_t* ids, const void* table, void* out,
                  int accumulate, void* stream) {
  tfm::EmbedGeo g;
  int rc = embed_check(e, g);
  if (rc) return rc;
  rc = rows_apart(e);
  if (rc) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (g.N == 0) return TFM_OK;
  if (!aligned(ids, 4) || !aligned(table, elem(e->table_dtype)) || !aligned(out, elem(e->dtype)))
    return fail(TFM_ERR_POINTER, "ids, table and out must be non-null and aligned to their "
                                 "elements");
  typedef tfm::bf16 bf16;
  if (e->table_dtype == TFM_BF16 && e->dtype == TFM_BF16)
    STEP("embed_fwd/hbm", tfm::launch_embed_fwd(g, ids, (const bf16*)table, (bf16*)out, accumulate, st));
  else if (e->table_dtype == TFM_BF16)
    STEP("embed_fwd/hbm", tfm::launch_embed_fwd(g, ids, (const bf16*)table, (float*)out, accumulate, st));
  else if (e->dtype == TFM_BF16)
    STEP("embed_fwd/hbm", tfm::launch_embed_fwd(g, ids, (const float*)table, (bf16*)out, accumulate, st));
  else
    STEP("embed_fwd/hbm", tfm::launch_embed_fwd(g, ids, (const float*)table, (float*)out, accumulate, st));
  return TFM_OK;
}

int tfm_embed_bwd(const tfm_embed* e, const int32_t* ids, const void* dout, float* dtable,
                  int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  tfm::EmbedGeo g;
  int rc = embed_check(e, g);
  if (rc) return rc;
  if ((g.N > 0 && (!aligned(ids, 4) || !aligned(dout, elem(e->dtype)))) || !aligned(dtable, 4))
    return fail(TFM_ERR_POINTER, "ids, dout and dtable must be non-null and aligned to their "
                                 "elements");
  if (!aligned(workspace, 16))
    return fail(TFM_ERR_POINTER, "workspace null or not 16-byte aligned");
  const size_t need = tfm::embed_bwd_bytes(g);
  if (workspace_bytes < need)
    return fail(TFM_ERR_BUFFER, "workspace has %zu bytes, %zu required", workspace_bytes, need);
  hipStream_t st = (hipStream_t)stream;
  if (g.N == 0 && accumulate) return TFM_OK;
  if (e->dtype == TFM_BF16)
    STEP("embed_bwd/hbm", tfm::launch_embed_bwd(g, ids, (const tfm::bf16*)dout, dtable, accumulate, workspace, st));
  else
    STEP("embed_bwd/hbm", tfm::launch_embed_bwd(g, ids, (const float*)dout, dtable, accumulate, workspace, st));
  return TFM_OK;
}

size_t tfm_distill_workspace_bytes(const tfm_distill* d) {
  if (distill_check(d)) return 0;
  return distill_ws(d).total;
}

int tfm_distill_loss(const tfm_distill* d, const void* logits, const int32_t* top_idx,
                     const float* top_logit, const float* top_lse, const int32_t* labels,
                     const float* weights, const int32_t* n_class, float* loss, float* row_loss,
                     void* dlogits, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = distill_check(d);
  if (rc) return rc;
  const size_t es = elem(d->dtype);
  if (!aligned(loss, 4) || !aligned_or_null(row_loss, 4))
    return fail(TFM_ERR_POINTER, "loss must be non-null and 4-byte aligned (row_loss too when "
                                 "given)");
  if (d->N > 0) {
    if (!aligned(logits, es) || !aligned(top_idx, 4) || !aligned(top_logit, 4) ||
        !aligned_or_null(dlogits, es))
      return fail(TFM_ERR_POINTER, "logits, top_idx and top_logit must be non-null and aligned to "
                                   "their elements (dlogits too when given)");
    if (d->tail && !aligned(top_lse, 4))
      return fail(TFM_ERR_POINTER, "tail = 1 needs top_lse, 4-byte aligned");
    if (d->alpha < 1.f && !labels)
      return fail(TFM_ERR_POINTER, "labels is null while alpha < 1");
    if (!aligned_or_null(labels, 4) || !aligned_or_null(weights, 4) || !aligned_or_null(n_class, 4))
      return fail(TFM_ERR_POINTER, "labels, weights and n_class must be 4-byte aligned");
    // dlogits is logits or lies apart from it
    const uintptr_t a = (uintptr_t)logits, b = (uintptr_t)dlogits;
    const uintptr_t span = ((uintptr_t)(d->N - 1) * d->ld + d->V) * es;
    if (dlogits && a != b && a < b + span && b < a + span)
      return fail(TFM_ERR_POINTER, "dlogits overlaps logits without being logits");
  }
  if (!aligned(workspace, 16))
    return fail(TFM_ERR_POINTER, "workspace null or not 16-byte aligned");
  const DistillWs W = distill_ws(d);
  if (workspace_bytes < W.total)
    return fail(TFM_ERR_BUFFER, "workspace has %zu bytes, %zu required", workspace_bytes, W.total);
  hipStream_t st = (hipStream_t)stream;
  tfm::DistillGeo g;
  g.N = d->N; g.ld = d->ld; g.V = d->V; g.k = d->k; g.tail = d->tail;
  g.tau = d->temperature; g.alpha = d->alpha;
  g.idx = top_idx; g.top = top_logit; g.lse = top_lse;
  g.labels = d->alpha < 1.f ? labels : nullptr;
  g.weights = weights; g.ncls = n_class;
  g.wsum = (double*)((char*)workspace + W.wsum);
  g.nwsum = 0;
  g.lsum = (double*)((char*)workspace + W.lsum);
  g.split = (char*)workspace + W.split;
  g.row_loss = row_loss ? row_loss : (float*)((char*)workspace + W.row_loss);
  if (weights && d->N > 0) STEP("distill_weights/hbm", tfm::launch_distill_weights(g, st));
  if (d->N > 0) {
    if (d->dtype == TFM_BF16)
      STEP("distill_rows/hbm", tfm::launch_distill_rows(g, (const tfm::bf16*)logits, (tfm::bf16*)dlogits, st));
    else
      STEP("distill_rows/hbm", tfm::launch_distill_rows(g, (const float*)logits, (float*)dlogits, st));
  }
  STEP("distill_loss/hbm", tfm::launch_distill_total(g, loss, st));
  return TFM_OK;
}

int tfm_sample(const tfm_sampling* s, const void* logits, const int32_t* n_class,
               const float* temperature, const int32_t* top_k, const float* top_p,
               const float* min_p, const float* u, int32_t* token, float* logprob, void* stream) {
  if (!s) return fail(TFM_ERR_POINTER, "the sampling's description is null");
  int rc = logits_check(s->N, s->V, s->dtype, s->ld);
  if (rc) return rc;
  if (s->N == 0) return TFM_OK;
  if (!aligned(logits, elem(s->dtype)) || !aligned(u, 4) || !aligned(token, 4))
    return fail(TFM_ERR_POINTER, "logits, u and token must be non-null and aligned to their "
                                 "elements");
  if (!aligned_or_null(n_class, 4) || !aligned_or_null(temperature, 4) ||
      !aligned_or_null(top_k, 4) || !aligned_or_null(top_p, 4) || !aligned_or_null(min_p, 4) ||
      !aligned_or_null(logprob, 4))
    return fail(TFM_ERR_POINTER, "n_class, temperature, top_k, top_p, min_p and logprob must be "
                                 "4-byte aligned");
  hipStream_t st = (hipStream_t)stream;
  tfm::SampleGeo g;
  g.N = s->N; g.ld = s->ld; g.V = s->V;
  g.ncls = n_class; g.temperature = temperature; g.top_k = top_k; g.top_p = top_p; g.min_p = min_p;
  g.u = u; g.token = token; g.logprob = logprob;
  if (s->dtype == TFM_BF16)
    STEP("sample/hbm", tfm::launch_sample(g, (const tfm::bf16*)logits, st));
  else
    STEP("sample/hbm", tfm::launch_sample(g, (const float*)logits, st));
  return TFM_OK;
}

}  // extern "C"
