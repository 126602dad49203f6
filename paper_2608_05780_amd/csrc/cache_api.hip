// C ABI of the key/value cache: argument checks and launches.
#include <algorithm>
#include <cmath>

#include "cache.h"

namespace {

using evisel::set_error;

evisel_status bad(const char* msg) {
  return set_error(EVISEL_ERR_INVALID_ARG, msg);
}

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// The view's own fields, and its device form.
evisel_status check_cache(const evisel_cache* c, evisel::CacheView* out) {
  if (!c) return bad("null cache");
  if (c->dtype != EVISEL_BF16 && c->dtype != EVISEL_FP32)
    return set_error(EVISEL_ERR_UNSUPPORTED, "dtype must be bf16 or fp32");
  if (c->d != 64 && c->d != 128)
    return set_error(EVISEL_ERR_UNSUPPORTED, "head dim must be 64 or 128");
  if (c->page < 16 || c->page > 1 << 20 || (c->page & (c->page - 1)))
    return set_error(EVISEL_ERR_UNSUPPORTED,
                     "page must be a power of two from 16 to 2^20");
  if (c->n_seq < 1 || c->hkv < 1 || c->max_pages < 1 || c->n_pages < 1)
    return bad("cache needs n_seq, hkv, max_pages and n_pages >= 1");
  if (c->n_pages > 0x7FFFFFFF) return bad("n_pages above 2^31 - 1");
  if (c->n_seq > 1 << 20 || c->hkv > 1 << 12)
    return bad("at most 2^20 sequences and 4096 kv heads");
  const int64_t cap = (int64_t)c->max_pages * c->page;
  if (cap > 1 << 30) return bad("capacity above 2^30 slots");
  if (!c->k || !c->v || !c->page_table || !c->length)
    return bad("null k, v, page_table or length");
  const int es = c->dtype == EVISEL_BF16 ? 2 : 4;
  if (!aligned(c->k, 16) || !aligned(c->v, 16))
    return bad("cache k and v must be 16-byte aligned");
  if (!aligned(c->page_table, 4) || !aligned(c->length, 4) ||
      !aligned(c->seen, 4) || !aligned(c->weight, 16) || !aligned(c->pos, 16))
    return bad("cache tables must be 4-byte, weight and pos 16-byte aligned");
  const int64_t ts = c->token_stride, hs = c->head_stride,
                ps = c->page_stride, most = 1 << 24;
  if (ts < c->d || hs < c->d || ps < c->d || ts > most || hs > most * c->page)
    return bad("cache strides out of range");
  if (ts * es % 16 || hs * es % 16 || ps * es % 16)
    return bad("cache strides must be multiples of 16 bytes");
  // rows of one page stay apart, and pages do, in either order of the axes
  const bool token_major = ts >= (int64_t)(c->hkv - 1) * hs + c->d;
  const bool head_major = hs >= (int64_t)(c->page - 1) * ts + c->d;
  if (!token_major && !head_major && c->hkv > 1)
    return bad("cache strides let rows overlap");
  if (c->n_pages > 1 &&
      ps < (int64_t)(c->page - 1) * ts + (int64_t)(c->hkv - 1) * hs + c->d)
    return bad("cache strides let pages overlap");
  if (ps > INT64_MAX / 8 / c->n_pages) return bad("cache strides out of range");
  evisel::CacheView& v = *out;
  v.k = (char*)c->k;
  v.v = (char*)c->v;
  v.table = c->page_table;
  v.length = c->length;
  v.seen = c->seen;
  v.weight = c->weight;
  v.pos = c->pos;
  v.n_pages = c->n_pages;
  v.page_bytes = ps * es;
  v.head_bytes = hs * es;
  v.token_bytes = (int32_t)(ts * es);
  v.n_seq = c->n_seq;
  v.hkv = c->hkv;
  v.d = c->d;
  v.page_shift = 0;
  while (1 << v.page_shift < c->page) ++v.page_shift;
  v.max_pages = c->max_pages;
  v.cap = cap;
  v.fp32 = c->dtype == EVISEL_FP32;
  return EVISEL_OK;
}

// Query heads of a kv head (the kernels' division by it is exact up to 2^13).
constexpr int kMaxGroup = 4096;

bool tree_bounds(const evisel::CacheView& c, int32_t hq, int32_t max_tree,
                 int32_t max_len) {
  return hq >= 1 && hq % c.hkv == 0 && hq / c.hkv <= kMaxGroup &&
         max_tree >= 1 &&
         max_tree <= 64 && max_len >= 0 && max_len <= c.cap;
}

}  // namespace

extern "C" {

evisel_status evisel_cache_append(const evisel_cache* cache,
                                  const void* k_new, const void* v_new,
                                  int32_t n_tok, const int32_t* tok_ptr,
                                  const int32_t* accept,
                                  const int32_t* n_accept, int32_t max_new,
                                  const float* w_new, void* stream) {
  evisel::CacheView c;
  const evisel_status st = check_cache(cache, &c);
  if (st != EVISEL_OK) return st;
  if (!c.seen) return bad("append needs the cache's seen");
  if (n_tok < 0 || max_new < 0) return bad("negative n_tok or max_new");
  if (!tok_ptr) return bad("null tok_ptr");
  if (n_tok == 0 || max_new == 0) return EVISEL_OK;
  if (!k_new || !v_new) return bad("null k_new or v_new");
  if (!aligned(k_new, 16) || !aligned(v_new, 16))
    return bad("k_new and v_new must be 16-byte aligned");
  if (!aligned(tok_ptr, 4) || !aligned(accept, 4) || !aligned(n_accept, 4) ||
      !aligned(w_new, 4))
    return bad("index and weight arrays must be 4-byte aligned");
  evisel::AppendCall a;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.tok_ptr = tok_ptr;
  a.accept = accept;
  a.n_accept = n_accept;
  a.w_new = w_new;
  a.n_tok = n_tok;
  a.max_new = std::min(max_new, n_tok);
  const hipError_t e = evisel::launch_cache_append(c, a, (hipStream_t)stream);
  if (e != hipSuccess) return evisel::set_hip_error(e, "cache append launch");
  return EVISEL_OK;
}

size_t evisel_tree_attention_workspace(const evisel_cache* cache, int32_t hq,
                                       int32_t max_tree, int32_t max_len,
                                       int32_t accumulate) {
  evisel::CacheView c;
  if (check_cache(cache, &c) != EVISEL_OK ||
      !tree_bounds(c, hq, max_tree, max_len))
    return 0;
  return evisel::plan_tree(c, hq, max_tree, max_len, accumulate != 0).total;
}

evisel_status evisel_tree_attention(
    const evisel_cache* cache, int32_t hq, const void* q, const void* k_new,
    const void* v_new, int32_t n_tok, const int32_t* tree_ptr,
    const int32_t* parent, int32_t max_tree, int32_t max_len,
    float softmax_scale, void* out, float* lse, int32_t accumulate,
    const float* vote, float decay, float* w_new, void* workspace,
    size_t workspace_bytes, void* stream) {
  evisel::CacheView c;
  const evisel_status st = check_cache(cache, &c);
  if (st != EVISEL_OK) return st;
  if (!tree_bounds(c, hq, max_tree, max_len))
    return bad("need hq a multiple of hkv (at most 4096 times it), "
               "1 <= max_tree <= 64 and 0 <= max_len <= capacity");
  if (n_tok < 0) return bad("negative n_tok");
  if (!tree_ptr) return bad("null tree_ptr");
  if ((k_new == nullptr) != (v_new == nullptr))
    return bad("k_new and v_new come together");
  if (!(softmax_scale > 0.f) || softmax_scale > 1e30f)
    return bad("softmax_scale must be positive");
  if (accumulate) {
    if (!c.weight) return bad("accumulate needs the cache's weight");
    if (!std::isfinite(decay)) return bad("decay must be finite");
  }
  if (n_tok == 0) return EVISEL_OK;
  if (!q || !out) return bad("null q or out");
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) ||
      !aligned(out, 16))
    return bad("q, k_new, v_new and out must be 16-byte aligned");
  if (!aligned(tree_ptr, 4) || !aligned(parent, 4) || !aligned(lse, 4) ||
      !aligned(vote, 4) || !aligned(w_new, 4))
    return bad("index, lse, vote and w_new arrays must be 4-byte aligned");
  const evisel::TreePlan p =
      evisel::plan_tree(c, hq, max_tree, max_len, accumulate != 0);
  if (p.total && (!workspace || workspace_bytes < p.total))
    return set_error(EVISEL_ERR_WORKSPACE,
                     "workspace smaller than evisel_tree_attention_workspace");
  if (!aligned(workspace, 256))
    return set_error(EVISEL_ERR_WORKSPACE,
                     "workspace must be 256-byte aligned");
  evisel::TreeCall t;
  t.q = (const char*)q;
  t.k_new = (const char*)k_new;
  t.v_new = (const char*)v_new;
  t.tree_ptr = tree_ptr;
  t.parent = parent;
  t.out = (char*)out;
  t.lse = lse;
  t.vote = accumulate ? vote : nullptr;
  t.w_new = accumulate ? w_new : nullptr;
  t.scale_log2 = softmax_scale * 1.4426950408889634f;
  const uint32_t group = (uint32_t)(hq / c.hkv);
  t.group_inv = group == 1 ? 0u : (uint32_t)(0xFFFFFFFFu / group) + 1u;
  t.decay = decay;
  t.hq = hq;
  t.n_tok = n_tok;
  t.max_tree = max_tree;
  t.max_len = max_len;
  t.accumulate = accumulate != 0;
  char* w = (char*)workspace;
  t.pO = (float*)(w + p.pO);
  t.pM = (float*)(w + p.pM);
  t.pL = (float*)(w + p.pL);
  t.share = (int32_t*)(w + p.share);
  t.row_m = (float*)(w + p.row_m);
  t.row_inv = (float*)(w + p.row_inv);
  t.score = (float*)(w + p.score);
  const hipError_t e =
      evisel::launch_tree_attention(c, p, t, (hipStream_t)stream);
  if (e != hipSuccess) return evisel::set_hip_error(e, "tree attention launch");
  return EVISEL_OK;
}

size_t evisel_cache_evict_workspace(const evisel_cache* cache, int32_t budget,
                                    int32_t max_len) {
  evisel::CacheView c;
  evisel::EvictCall e;
  if (check_cache(cache, &c) != EVISEL_OK || budget < 1 || max_len < 0 ||
      max_len > c.cap)
    return 0;
  e.budget = budget;
  e.max_len = max_len;
  return evisel::evict_layout(c, e, nullptr);
}

evisel_status evisel_cache_evict(const evisel_cache* cache, int32_t budget,
                                 int32_t n_sink, int32_t n_recent,
                                 int32_t max_len, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  evisel::CacheView c;
  const evisel_status st = check_cache(cache, &c);
  if (st != EVISEL_OK) return st;
  if (!c.seen || !c.weight || !c.pos)
    return bad("evict needs the cache's seen, weight and pos");
  if (budget < 1 || n_sink < 0 || n_recent < 0 ||
      (int64_t)n_sink + n_recent > budget)
    return bad("need budget >= 1 and 0 <= n_sink + n_recent <= budget");
  if (max_len < 0 || max_len > c.cap)
    return bad("need 0 <= max_len <= capacity");
  evisel::EvictCall e;
  e.budget = budget;
  e.n_sink = n_sink;
  e.n_recent = n_recent;
  e.max_len = max_len;
  const size_t need = evisel::evict_layout(c, e, (char*)workspace);
  if (e.max_moves == 0) return EVISEL_OK;   // no sequence is over the budget
  if (!workspace || workspace_bytes < need)
    return set_error(EVISEL_ERR_WORKSPACE,
                     "workspace smaller than evisel_cache_evict_workspace");
  if (!aligned(workspace, 256))
    return set_error(EVISEL_ERR_WORKSPACE,
                     "workspace must be 256-byte aligned");
  const hipError_t err =
      evisel::launch_cache_evict(c, e, (hipStream_t)stream);
  if (err != hipSuccess) return evisel::set_hip_error(err, "cache evict launch");
  return EVISEL_OK;
}

}  // extern "C"
