// Host side of the decode entry points of the C ABI (paged cache, sampling, embedding rows): argument
// validation (all of it before the first HIP call), workspace planning and kernel sequencing.
#include <stdarg.h>
#include <stdio.h>

#include "../../include/zo.h"
#include "zo_host.hpp"
#include "zo_internal.hpp"

namespace {

int32_t fail(zo_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return zo::fail_status(st, buf);
}

#define ZO_HIP(call, where)                                                                       \
  do {                                                                                            \
    hipError_t e__ = (call);                                                                      \
    if (e__ != hipSuccess) return fail(ZO_ERR_HIP, "%s: %s", where, hipGetErrorString(e__));      \
  } while (0)

constexpr int64_t kMaxLd = (int64_t)1 << 22;
constexpr int64_t kMaxThreads = (int64_t)1 << 31;   // of a launch along one dimension
constexpr int kMaxVocab = 1 << 19;   // (2^44 per weight of 64-bit bin sums)

int32_t check_cache(const zo_batch* b, const zo_cache* c) {
  if (!c) return fail(ZO_ERR_NULL, "cache is NULL");
  if (c->dtype != ZO_F32 && c->dtype != ZO_BF16) return fail(ZO_ERR_UNSUPPORTED, "cache dtype %d", (int)c->dtype);
  if (c->n_pages < 1 || c->max_pages < 1 || c->n_kv_heads < 1 || c->head_dim < 1)
    return fail(ZO_ERR_SHAPE, "cache n_pages = %d, max_pages = %d, n_kv_heads = %d, head_dim = %d", c->n_pages,
                c->max_pages, c->n_kv_heads, c->head_dim);
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return fail(ZO_ERR_UNSUPPORTED, "cache page_size = %d: powers of two from 16 to 1024 are covered", c->page_size);
  const int64_t cap = (int64_t)c->max_pages * c->page_size;
  if (cap > (int64_t)1 << 30) return fail(ZO_ERR_SHAPE, "cache max_pages * page_size = %lld exceeds 2^30", (long long)cap);
  if ((int64_t)c->n_kv_heads * c->head_dim > kMaxLd) return fail(ZO_ERR_SHAPE, "n_kv_heads * head_dim too large");
  if (!c->K || !c->V) return fail(ZO_ERR_NULL, "cache.K / cache.V is NULL");
  if ((((uintptr_t)c->K | (uintptr_t)c->V) & 15u) != 0) return fail(ZO_ERR_SHAPE, "cache.K / cache.V not 16-byte aligned");
  if (b->n_seqs > 0 && (!c->page_table || !c->kv_len)) return fail(ZO_ERR_NULL, "cache.page_table / cache.kv_len is NULL");
  if (c->host_kv_len)
    for (int s = 0; s < b->n_seqs; ++s) {
      const int32_t n = c->host_kv_len[s];
      const int rows = b->host_cu_seqlens ? b->host_cu_seqlens[s + 1] - b->host_cu_seqlens[s] : 0;
      if (n < rows || n > cap)
        return fail(ZO_ERR_INDEX, "kv_len[%d] = %d outside [%d, %lld] (its rows, its pages)", s, n, rows, (long long)cap);
      if (c->host_page_table)
        for (int j = 0; j < (n + c->page_size - 1) / c->page_size; ++j) {
          const int32_t pg = c->host_page_table[(int64_t)s * c->max_pages + j];
          if (pg < 0 || pg >= c->n_pages)
            return fail(ZO_ERR_INDEX, "page_table[%d][%d] = %d outside [0, %d)", s, j, pg, c->n_pages);
        }
    }
  return ZO_OK;
}

int32_t check_heads(int32_t n_heads, const zo_cache* c) {
  if (n_heads < 1 || n_heads > 65535) return fail(ZO_ERR_SHAPE, "n_heads = %d", n_heads);
  if (n_heads % c->n_kv_heads != 0)
    return fail(ZO_ERR_SHAPE, "n_heads = %d is not a multiple of n_kv_heads = %d", n_heads, c->n_kv_heads);
  if ((int64_t)n_heads * c->head_dim > kMaxLd) return fail(ZO_ERR_SHAPE, "n_heads * head_dim too large");
  return ZO_OK;
}

zo::CacheDev to_dev(const zo_cache* c) {
  zo::CacheDev d;
  d.K = c->K; d.V = c->V; d.table = c->page_table; d.kv_len = c->kv_len;
  d.n_pages = c->n_pages; d.max_pages = c->max_pages; d.n_kv_heads = c->n_kv_heads; d.dh = c->head_dim;
  d.bf16 = c->dtype == ZO_BF16;
  d.page_shift = 0;
  while ((1 << d.page_shift) < c->page_size) ++d.page_shift;
  return d;
}

// Whether `items` times the threads of each fit one launch.
int32_t check_launch(const char* what, int64_t items, int64_t threads) {
  if (items > kMaxThreads / threads) return fail(ZO_ERR_UNSUPPORTED, "%s = %lld: up to %lld fit one call", what, (long long)items, (long long)(kMaxThreads / threads));
  return ZO_OK;
}

// A matrix of rows that need no alignment beyond their type's.
int32_t check_rows(const char* name, const void* p, int64_t ld, int cols, zo_dtype dt) {
  if (ld < cols || ld > kMaxLd)
    return fail(ZO_ERR_SHAPE, "%s: leading dimension %lld invalid for %d columns", name, (long long)ld, cols);
  if (((uintptr_t)p & (dt == ZO_BF16 ? 1u : 3u)) != 0) return fail(ZO_ERR_SHAPE, "%s: pointer misaligned", name);
  return ZO_OK;
}

int32_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return ZO_OK;
  if (!ws) return fail(ZO_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  if (((uintptr_t)ws & 255u) != 0) return fail(ZO_ERR_WORKSPACE, "workspace not 256-byte aligned");
  if (have < need) return fail(ZO_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return ZO_OK;
}

// Partial results of the ranges of long rows; nothing when every row is one range.
struct PagedPlan {
  int ranges = 1;
  size_t ml = 0, o = 0, total = 0;
};
PagedPlan plan_paged(int T, int H, int dh, int max_len, zo_dtype dt) {
  PagedPlan p;
  p.ranges = zo::attention_paged_ranges(dt == ZO_BF16, max_len);
  if (p.ranges > 1) {
    const size_t parts = (size_t)T * H * p.ranges;
    p.o = (parts * 8 + 255) / 256 * 256;
    p.total = p.o + (parts * dh * 4 + 255) / 256 * 256;
  }
  return p;
}

}  // namespace

extern "C" {

int32_t zo_cache_append(const zo_batch* batch, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V,
                        int64_t ldv, int32_t n_heads, const float* gamma_q, const float* gamma_k, float norm_eps,
                        float rope_theta, const zo_cache* cache, void* Qout, int64_t ldqo, void* stream) {
  if (int32_t st = zo::batch_validate(batch)) return st;
  if (int32_t st = check_cache(batch, cache)) return st;
  if (int32_t st = check_heads(n_heads, cache)) return st;
  const int dh = cache->head_dim;
  if (dh % 2 != 0 || dh > 256) return fail(ZO_ERR_UNSUPPORTED, "head_dim = %d: even values up to 256 are covered", dh);
  if ((gamma_q == nullptr) != (gamma_k == nullptr)) return fail(ZO_ERR_NULL, "gamma_q and gamma_k go together");
  if ((((uintptr_t)gamma_q | (uintptr_t)gamma_k) & 3u) != 0) return fail(ZO_ERR_SHAPE, "gamma_q / gamma_k: pointer misaligned");
  if (!(norm_eps >= 0.0f)) return fail(ZO_ERR_SHAPE, "norm_eps = %g", (double)norm_eps);
  if (batch->n_tokens == 0) return ZO_OK;
  if (int32_t st = check_launch("n_tokens * (n_heads + 2 * n_kv_heads)", (int64_t)batch->n_tokens * (n_heads + 2 * cache->n_kv_heads), 64)) return st;
  if (!Q || !K || !V || !Qout) return fail(ZO_ERR_NULL, "Q, K, V or Qout is NULL");
  if (Qout == Q && ldqo != ldq) return fail(ZO_ERR_SHAPE, "Qout is Q, but with another leading dimension");
  const zo_dtype dt = cache->dtype;
  if (int32_t st = zo::matrix_validate("Q", Q, ldq, n_heads * dh, dt)) return st;
  if (int32_t st = zo::matrix_validate("K", K, ldk, cache->n_kv_heads * dh, dt)) return st;
  if (int32_t st = zo::matrix_validate("V", V, ldv, cache->n_kv_heads * dh, dt)) return st;
  if (int32_t st = zo::matrix_validate("Qout", Qout, ldqo, n_heads * dh, dt)) return st;
  zo::AppendArgs a;
  a.Q = Q; a.ldq = ldq; a.K = K; a.ldk = ldk; a.V = V; a.ldv = ldv; a.Qout = Qout; a.ldqo = ldqo;
  a.cu = batch->cu_seqlens; a.S = batch->n_seqs; a.T = batch->n_tokens; a.n_heads = n_heads;
  a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.eps = norm_eps; a.theta = rope_theta > 0.0f ? rope_theta : 0.0f;
  a.c = to_dev(cache);
  if (Qout == Q && !gamma_q && a.theta == 0.0f) a.n_heads = 0;   // (queries that stay as and where they are)
  ZO_HIP(zo::launch_cache_append(a, (hipStream_t)stream), "zo_cache_append");
  return ZO_OK;
}

size_t zo_attention_paged_workspace_bytes(int32_t n_tokens, int32_t n_heads, int32_t head_dim, int32_t max_len,
                                          zo_dtype dtype) {
  if (n_tokens < 0 || n_heads < 0 || head_dim < 0 || max_len < 0) return 0;
  return plan_paged(n_tokens, n_heads, head_dim, max_len, dtype).total;
}

int32_t zo_attention_paged(const zo_batch* batch, const void* Q, int64_t ldq, int32_t n_heads, float scale,
                           const zo_cache* cache, void* O, int64_t ldo, void* workspace, size_t workspace_bytes,
                           void* stream) {
  if (int32_t st = zo::batch_validate(batch)) return st;
  if (int32_t st = check_cache(batch, cache)) return st;
  if (int32_t st = check_heads(n_heads, cache)) return st;
  const int dh = cache->head_dim;
  const zo_dtype dt = cache->dtype;
  if (dt == ZO_BF16 && dh != 64 && dh != 128 && dh != 256)
    return fail(ZO_ERR_UNSUPPORTED, "the bf16 kernel covers head_dim 64, 128 and 256 (head_dim = %d)", dh);
  if (dh > 256) return fail(ZO_ERR_UNSUPPORTED, "the fp32 kernel covers head_dim <= 256 (head_dim = %d)", dh);
  const int T = batch->n_tokens;
  if (T == 0) return ZO_OK;
  if (int32_t st = check_launch("n_tokens * n_heads", (int64_t)T * n_heads, 256)) return st;
  if (!Q || !O) return fail(ZO_ERR_NULL, "Q or O is NULL");
  if (int32_t st = zo::matrix_validate("Q", Q, ldq, n_heads * dh, dt)) return st;
  if (int32_t st = zo::matrix_validate("O", O, ldo, n_heads * dh, dt)) return st;
  const PagedPlan plan = plan_paged(T, n_heads, dh, cache->max_pages * cache->page_size, dt);
  if (int32_t st = check_workspace(workspace, workspace_bytes, plan.total)) return st;
  zo::PagedAttnArgs a;
  a.Q = Q; a.ldq = ldq; a.O = O; a.ldo = ldo; a.cu = batch->cu_seqlens; a.S = batch->n_seqs; a.T = T;
  a.n_heads = n_heads; a.group = n_heads / cache->n_kv_heads; a.scale = scale; a.c = to_dev(cache);
  a.ranges = plan.ranges;
  a.part_ml = plan.ranges > 1 ? (float*)((char*)workspace + plan.ml) : nullptr;
  a.part_o = plan.ranges > 1 ? (float*)((char*)workspace + plan.o) : nullptr;
  ZO_HIP(zo::launch_attention_paged(a, (hipStream_t)stream), "zo_attention_paged");
  return ZO_OK;
}

size_t zo_sample_workspace_bytes(int32_t n_rows, int32_t vocab, zo_dtype dtype) {
  (void)n_rows; (void)vocab; (void)dtype;
  return 0;
}

int32_t zo_sample(const void* logits, int64_t ld, int32_t n_rows, int32_t vocab, zo_dtype dtype,
                  const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                  int32_t* tokens, float* prob, int32_t* n_kept, void* workspace, size_t workspace_bytes, void* stream) {
  if (n_rows < 0 || vocab < 1) return fail(ZO_ERR_SHAPE, "n_rows = %d, vocab = %d", n_rows, vocab);
  if (vocab > kMaxVocab) return fail(ZO_ERR_UNSUPPORTED, "vocab = %d: up to %d are covered", vocab, kMaxVocab);
  if (dtype != ZO_F32 && dtype != ZO_BF16) return fail(ZO_ERR_UNSUPPORTED, "dtype %d", (int)dtype);
  if (n_rows == 0) return ZO_OK;
  if (int32_t st = check_launch("n_rows", n_rows, 1024)) return st;
  if (!logits || !temperature || !u || !tokens) return fail(ZO_ERR_NULL, "logits, temperature, u or tokens is NULL");
  if (int32_t st = check_rows("logits", logits, ld, vocab, dtype)) return st;
  if (int32_t st = check_workspace(workspace, workspace_bytes, zo_sample_workspace_bytes(n_rows, vocab, dtype))) return st;
  zo::SampleArgs a;
  a.z = logits; a.ld = ld; a.T = n_rows; a.V = vocab; a.bf16 = dtype == ZO_BF16;
  a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u;
  a.tokens = tokens; a.prob = prob; a.n_kept = n_kept;
  ZO_HIP(zo::launch_sample(a, (hipStream_t)stream), "zo_sample");
  return ZO_OK;
}

int32_t zo_embed_rows(const int32_t* tokens, const int32_t* pos, int32_t n_rows, const void* E, int64_t lde,
                      int32_t vocab, const void* E_pos, int64_t ldp, int32_t n_pos, int32_t d, zo_dtype dtype, void* X,
                      int64_t ldx, int32_t* pos_next, void* stream) {
  if (n_rows < 0 || vocab < 0 || n_pos < 0 || d < 0)
    return fail(ZO_ERR_SHAPE, "n_rows = %d, vocab = %d, n_pos = %d, d = %d", n_rows, vocab, n_pos, d);
  if (dtype != ZO_F32 && dtype != ZO_BF16) return fail(ZO_ERR_UNSUPPORTED, "dtype %d", (int)dtype);
  if (n_rows == 0) return ZO_OK;
  if (int32_t st = check_launch("n_rows", n_rows, 256)) return st;
  if (!tokens) return fail(ZO_ERR_NULL, "tokens is NULL");
  if (!pos && (E_pos || pos_next)) return fail(ZO_ERR_NULL, "pos is NULL");
  if (d > 0) {
    if (!E || !X) return fail(ZO_ERR_NULL, "E or X is NULL");
    if (int32_t st = check_rows("E", E, lde, d, dtype)) return st;
    if (E_pos)
      if (int32_t st = check_rows("E_pos", E_pos, ldp, d, dtype)) return st;
    if (int32_t st = check_rows("X", X, ldx, d, dtype)) return st;
  }
  zo::EmbedArgs a;
  a.tokens = tokens; a.pos = pos; a.T = n_rows; a.E = E; a.lde = lde; a.vocab = vocab; a.Epos = E_pos; a.ldp = ldp;
  a.n_pos = n_pos; a.d = d; a.bf16 = dtype == ZO_BF16; a.X = X; a.ldx = ldx; a.pos_next = pos_next;
  ZO_HIP(zo::launch_embed_rows(a, (hipStream_t)stream), "zo_embed_rows");
  return ZO_OK;
}

}  // extern "C"
