// C-ABI entry points of the cache and attention operators: argument checks
// on the host, then kernel launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "attention.h"
#include "s2moe.h"
#include "status.h"

static_assert(s2moe::kKvMaxRequests == S2MOE_KV_MAX_REQUESTS, "request limit");
static_assert(s2moe::kMaxNodes == S2MOE_MAX_TOKENS, "tree limit");
static_assert((int)s2moe::kKvNoPages == (int)S2MOE_KV_NO_PAGES &&
                  (int)s2moe::kKvTooLong == (int)S2MOE_KV_TOO_LONG &&
                  (int)s2moe::kKvBadSeq == (int)S2MOE_KV_BAD_SEQ &&
                  (int)s2moe::kKvBusy == (int)S2MOE_KV_BUSY &&
                  (int)s2moe::kKvBadPath == (int)S2MOE_KV_BAD_PATH,
              "status bits");

namespace {

using s2moe::aligned;
using s2moe::aligned16;
using s2moe::fail;
using s2moe::hip_status;
using s2moe::ok;

// Integer arrays may start anywhere a 32-bit integer may.
#define S2MOE_REQUIRE_INTS(p)                                                              \
  do {                                                                                     \
    if ((p) == nullptr) return fail(S2MOE_EINVAL, "%s: %s is NULL", fn, #p);               \
    if (!aligned(p, 4)) return fail(S2MOE_EINVAL, "%s: %s is not 4-byte aligned", fn, #p); \
  } while (0)

s2moe_status check_cache(const char* fn, const s2moe_kv_cache* cache, s2moe::KvCache* out) {
  if (cache == nullptr) return fail(S2MOE_EINVAL, "%s: cache is NULL", fn);
  const s2moe_kv_cache& c = *cache;
  if (c.dtype != S2MOE_F32 && c.dtype != S2MOE_BF16)
    return fail(S2MOE_EINVAL, "%s: dtype = %d must be F32 or BF16", fn, c.dtype);
  if (c.head_dim != 64 && c.head_dim != 128)
    return fail(c.head_dim < 1 ? S2MOE_EINVAL : S2MOE_EUNSUPPORTED,
                "%s: head_dim = %d must be 64 or 128", fn, c.head_dim);
  if (c.n_kv_heads < 1) return fail(S2MOE_EINVAL, "%s: n_kv_heads = %d < 1", fn, c.n_kv_heads);
  if (c.n_kv_heads > 256)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_kv_heads = %d exceeds 256", fn, c.n_kv_heads);
  if (c.n_layers < 1) return fail(S2MOE_EINVAL, "%s: n_layers = %d < 1", fn, c.n_layers);
  if (c.n_layers > 1024)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_layers = %d exceeds 1024", fn, c.n_layers);
  if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128 &&
      c.page_size != 256)
    return fail(S2MOE_EINVAL, "%s: page_size = %d must be 16, 32, 64, 128 or 256", fn,
                c.page_size);
  if (c.n_pages < 1 || c.n_pages > (1 << 24))
    return fail(S2MOE_EINVAL, "%s: n_pages = %d not in [1, 2^24]", fn, c.n_pages);
  if (c.max_seqs < 1 || c.max_seqs > (1 << 20))
    return fail(S2MOE_EINVAL, "%s: max_seqs = %d not in [1, 2^20]", fn, c.max_seqs);
  if (c.max_pages < 1 || (int64_t)c.max_pages * c.page_size >= (int64_t)1 << 31)
    return fail(S2MOE_EINVAL, "%s: max_pages = %d pages of %d tokens not in [1, 2^31) tokens", fn,
                c.max_pages, c.page_size);
  S2MOE_REQUIRE_PTR(c.k);
  S2MOE_REQUIRE_PTR(c.v);
  S2MOE_REQUIRE_INTS(c.table);
  S2MOE_REQUIRE_INTS(c.length);
  S2MOE_REQUIRE_INTS(c.refs);
  s2moe::KvCache& o = *out;
  o.L = c.n_layers;
  o.Hkv = c.n_kv_heads;
  o.D = c.head_dim;
  o.n_pages = c.n_pages;
  o.P = c.page_size;
  o.log_p = __builtin_ctz((unsigned)c.page_size);
  o.max_seqs = c.max_seqs;
  o.max_pages = c.max_pages;
  o.f32 = c.dtype == S2MOE_F32;
  o.k = static_cast<char*>(c.k);
  o.v = static_cast<char*>(c.v);
  o.table = c.table;
  o.length = c.length;
  o.refs = c.refs;
  return S2MOE_OK;
}

s2moe_status check_requests(const char* fn, int32_t n) {
  if (n < 0) return fail(S2MOE_EINVAL, "%s: n = %d < 0", fn, n);
  if (n > S2MOE_KV_MAX_REQUESTS)
    return fail(S2MOE_EUNSUPPORTED, "%s: n = %d exceeds %d", fn, n, S2MOE_KV_MAX_REQUESTS);
  return S2MOE_OK;
}

s2moe_status check_layer_index(const char* fn, const s2moe::KvCache& c, int32_t layer) {
  if (layer < 0 || layer >= c.L)
    return fail(S2MOE_EINVAL, "%s: layer = %d not in [0, %d)", fn, layer, c.L);
  return S2MOE_OK;
}

// Rows of `heads` heads, `ld` elements apart.
s2moe_status check_rows(const char* fn, const char* name, int64_t ld, int heads, int D, int elt) {
  if (ld < (int64_t)heads * D)
    return fail(S2MOE_EINVAL, "%s: %s = %lld must be at least %d heads of %d", fn, name,
                (long long)ld, heads, D);
  if (ld > (int64_t)1 << 22)
    return fail(S2MOE_EUNSUPPORTED, "%s: %s = %lld exceeds 2^22 elements", fn, name, (long long)ld);
  if (ld * elt % 16 != 0)
    return fail(S2MOE_EINVAL, "%s: %s = %lld elements is not a multiple of 16 bytes", fn, name,
                (long long)ld);
  return S2MOE_OK;
}

// Whether rows of wa bytes every lda meet rows of wb bytes every ldb (n rows
// each): rows of one wider array may lie side by side.
bool rows_meet(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb,
               int64_t n) {
  const int64_t x = (int64_t)reinterpret_cast<uintptr_t>(a);
  const int64_t y = (int64_t)reinterpret_cast<uintptr_t>(b);
  if (y >= x + (n - 1) * lda + wa || x >= y + (n - 1) * ldb + wb) return false;
  if (lda != ldb) return true;
  const int64_t at = ((y - x) % lda + lda) % lda;  // where b's rows start within a's period
  return at < wa || at + wb > lda;
}

s2moe_status check_attn(const char* fn, const s2moe_attn* attn) {
  if (attn == nullptr) return fail(S2MOE_EINVAL, "%s: attn is NULL", fn);
  const s2moe_attn& t = *attn;
  if (t.dtype != S2MOE_F32 && t.dtype != S2MOE_BF16)
    return fail(S2MOE_EINVAL, "%s: dtype = %d must be F32 or BF16", fn, t.dtype);
  if (t.head_dim != 64 && t.head_dim != 128)
    return fail(t.head_dim < 1 ? S2MOE_EINVAL : S2MOE_EUNSUPPORTED,
                "%s: head_dim = %d must be 64 or 128", fn, t.head_dim);
  if (t.n_kv_heads < 1 || t.n_heads < 1 || t.n_heads % t.n_kv_heads != 0)
    return fail(S2MOE_EINVAL, "%s: n_heads = %d must be a positive multiple of n_kv_heads = %d",
                fn, t.n_heads, t.n_kv_heads);
  if (t.n_heads > 1024 || t.n_kv_heads > 256)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_heads = %d, n_kv_heads = %d exceed 1024, 256", fn,
                t.n_heads, t.n_kv_heads);
  if (!std::isfinite(t.scale) || !(t.scale > 0.f))
    return fail(S2MOE_EINVAL, "%s: scale = %g must be finite and > 0", fn, (double)t.scale);
  return S2MOE_OK;
}

s2moe_status check_tree(const char* fn, const s2moe_kv_cache* cache, const s2moe_attn* attn,
                        int32_t n, int32_t max_nodes, s2moe::KvCache* c) {
  s2moe_status st = check_cache(fn, cache, c);
  if (st == S2MOE_OK) st = check_attn(fn, attn);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (attn->n_kv_heads != c->Hkv || attn->head_dim != c->D || (attn->dtype == S2MOE_F32) != c->f32)
    return fail(S2MOE_EINVAL, "%s: n_kv_heads, head_dim and dtype of attn differ from the cache's",
                fn);
  if (max_nodes < 1) return fail(S2MOE_EINVAL, "%s: max_nodes = %d < 1", fn, max_nodes);
  if (max_nodes > S2MOE_MAX_TOKENS)
    return fail(S2MOE_EUNSUPPORTED, "%s: max_nodes = %d exceeds %d", fn, max_nodes,
                S2MOE_MAX_TOKENS);
  // Units of work of one sequence: a 32-bit number on the device.
  const int64_t tiles = (int64_t)c->max_pages * c->P / 128 + 1;
  const int64_t blocks = ((int64_t)attn->n_heads / c->Hkv * max_nodes + 15) / 16;
  if (tiles * blocks * c->Hkv >= (int64_t)1 << 31)
    return fail(S2MOE_EUNSUPPORTED, "%s: sequences of up to %d pages with %d heads and %d nodes", fn,
                c->max_pages, attn->n_heads, max_nodes);
  return S2MOE_OK;
}

// The part of a tree attention call that its workspace depends on.
void tree_sizes(const s2moe::KvCache& c, const s2moe_attn* attn, int32_t max_nodes,
                s2moe::TreeArgs* a) {
  a->Hq = attn->n_heads;
  a->Hkv = c.Hkv;
  a->G = attn->n_heads / c.Hkv;
  a->D = c.D;
  a->f32 = c.f32;
  a->max_nodes = max_nodes;
}

}  // namespace

extern "C" {

s2moe_status s2moe_kv_init(const s2moe_kv_cache* cache, void* stream) {
  const char* fn = "s2moe_kv_init";
  s2moe::KvCache c;
  const s2moe_status st = check_cache(fn, cache, &c);
  if (st != S2MOE_OK) return st;
  return hip_status(fn, s2moe::launch_kv_init(c, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_fork(const s2moe_kv_cache* cache, int32_t n, const int32_t* src,
                           const int32_t* dst, int32_t* status, void* stream) {
  const char* fn = "s2moe_kv_fork";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (n == 0) return ok();
  S2MOE_REQUIRE_INTS(src);
  S2MOE_REQUIRE_INTS(dst);
  S2MOE_REQUIRE_INTS(status);
  return hip_status(fn, s2moe::launch_kv_fork(c, n, src, dst, status,
                                              static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_reserve(const s2moe_kv_cache* cache, int32_t n, const int32_t* seqs,
                              const int32_t* extra, int32_t* copied, int32_t* status,
                              void* stream) {
  const char* fn = "s2moe_kv_reserve";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (n == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(extra);
  S2MOE_REQUIRE_INTS(copied);
  S2MOE_REQUIRE_INTS(status);
  return hip_status(fn, s2moe::launch_kv_reserve(c, n, seqs, extra, copied, status,
                                                 static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_append(const s2moe_kv_cache* cache, int32_t layer, int32_t n,
                             int32_t n_tokens, const int32_t* seqs, const int32_t* tok_off,
                             const void* k, int64_t ldk, const void* v, int64_t ldv,
                             void* stream) {
  const char* fn = "s2moe_kv_append";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st == S2MOE_OK) st = check_layer_index(fn, c, layer);
  if (st != S2MOE_OK) return st;
  if (n_tokens < 0) return fail(S2MOE_EINVAL, "%s: n_tokens = %d < 0", fn, n_tokens);
  if (n == 0 || n_tokens == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(tok_off);
  S2MOE_REQUIRE_PTR(k);
  S2MOE_REQUIRE_PTR(v);
  if ((st = check_rows(fn, "ldk", ldk, c.Hkv, c.D, c.elt())) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldv", ldv, c.Hkv, c.D, c.elt())) != S2MOE_OK) return st;
  s2moe::AppendArgs a;
  a.layer = layer;
  a.n = n;
  a.n_tokens = n_tokens;
  a.seqs = seqs;
  a.tok_off = tok_off;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.ldk = ldk;
  a.ldv = ldv;
  return hip_status(fn, s2moe::launch_kv_append(c, a, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_commit(const s2moe_kv_cache* cache, int32_t n, int32_t max_path,
                             const int32_t* seqs, const int32_t* path, const int32_t* n_accept,
                             int32_t* status, void* stream) {
  const char* fn = "s2moe_kv_commit";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (max_path < 0) return fail(S2MOE_EINVAL, "%s: max_path = %d < 0", fn, max_path);
  if (max_path > S2MOE_MAX_TOKENS)
    return fail(S2MOE_EUNSUPPORTED, "%s: max_path = %d exceeds %d", fn, max_path,
                S2MOE_MAX_TOKENS);
  if (n == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(n_accept);
  S2MOE_REQUIRE_INTS(status);
  if (path != nullptr && !aligned(path, 4))
    return fail(S2MOE_EINVAL, "%s: path is not 4-byte aligned", fn);
  return hip_status(fn, s2moe::launch_kv_commit(c, n, max_path, seqs, path, n_accept, status,
                                                static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_free(const s2moe_kv_cache* cache, int32_t n, const int32_t* seqs,
                           int32_t* status, void* stream) {
  const char* fn = "s2moe_kv_free";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (n == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(status);
  return hip_status(fn,
                    s2moe::launch_kv_free(c, n, seqs, status, static_cast<hipStream_t>(stream)));
}

size_t s2moe_tree_attention_workspace_bytes(const s2moe_kv_cache* cache, const s2moe_attn* attn,
                                            int32_t n, int32_t max_nodes) {
  s2moe::KvCache c;
  if (check_tree("s2moe_tree_attention_workspace_bytes", cache, attn, n, max_nodes, &c) !=
      S2MOE_OK)
    return 0;
  s2moe::TreeArgs a{};
  tree_sizes(c, attn, max_nodes, &a);
  return s2moe::tree_attention_workspace(a);
}

s2moe_status s2moe_tree_attention(const s2moe_kv_cache* cache, int32_t layer,
                                  const s2moe_attn* attn, int32_t n, int32_t n_tokens,
                                  int32_t max_nodes, const void* q, const int32_t* seqs,
                                  const int32_t* tok_off, const int32_t* parent, void* workspace,
                                  size_t workspace_bytes, void* out, void* stream) {
  const char* fn = "s2moe_tree_attention";
  s2moe::KvCache c;
  s2moe_status st = check_tree(fn, cache, attn, n, max_nodes, &c);
  if (st == S2MOE_OK) st = check_layer_index(fn, c, layer);
  if (st != S2MOE_OK) return st;
  if (n_tokens < 0) return fail(S2MOE_EINVAL, "%s: n_tokens = %d < 0", fn, n_tokens);
  if (n == 0 || n_tokens == 0) return ok();
  S2MOE_REQUIRE_PTR(q);
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(tok_off);
  S2MOE_REQUIRE_INTS(parent);
  S2MOE_REQUIRE_PTR(out);
  const int Hq = attn->n_heads, elt = c.elt();
  if ((st = check_rows(fn, "ldq", attn->ldq, Hq, c.D, elt)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldo", attn->ldo, Hq, c.D, elt)) != S2MOE_OK) return st;
  const int64_t w = (int64_t)Hq * c.D * elt;
  if (rows_meet(q, attn->ldq * elt, w, out, attn->ldo * elt, w, n_tokens))
    return fail(S2MOE_EINVAL, "%s: out overlaps q", fn);
  s2moe::TreeArgs a{};
  tree_sizes(c, attn, max_nodes, &a);
  const size_t need = s2moe::tree_attention_workspace(a);
  if (workspace == nullptr)
    return fail(S2MOE_EWORKSPACE, "%s: workspace is NULL (%zu bytes needed)", fn, need);
  if (!aligned16(workspace))
    return fail(S2MOE_EINVAL, "%s: workspace is not 16-byte aligned", fn);
  if (workspace_bytes < need)
    return fail(S2MOE_EWORKSPACE, "%s: workspace holds %zu bytes, %zu needed", fn,
                workspace_bytes, need);
  a.k = c.k + layer * c.layer_bytes();
  a.v = c.v + layer * c.layer_bytes();
  a.table = c.table;
  a.length = c.length;
  a.n_pages = c.n_pages;
  a.P = c.P;
  a.log_p = c.log_p;
  a.max_seqs = c.max_seqs;
  a.max_pages = c.max_pages;
  a.n = n;
  a.n_tokens = n_tokens;
  a.seqs = seqs;
  a.tok_off = tok_off;
  a.parent = parent;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.ldq = attn->ldq;
  a.ldo = attn->ldo;
  a.scale = attn->scale;
  a.ws = static_cast<float*>(workspace);
  return hip_status(fn, s2moe::launch_tree_attention(a, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_prompt_attention(const s2moe_attn* attn, int32_t n, int32_t n_tokens,
                                    const void* q, const void* k, const void* v,
                                    const int32_t* tok_off, void* out, void* stream) {
  const char* fn = "s2moe_prompt_attention";
  s2moe_status st = check_attn(fn, attn);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st != S2MOE_OK) return st;
  if (n_tokens < 0) return fail(S2MOE_EINVAL, "%s: n_tokens = %d < 0", fn, n_tokens);
  if ((int64_t)n_tokens * attn->n_heads >= (int64_t)1 << 31)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_tokens = %d of %d heads: 2^31 rows or more", fn,
                n_tokens, attn->n_heads);
  if (n == 0 || n_tokens == 0) return ok();
  S2MOE_REQUIRE_PTR(q);
  S2MOE_REQUIRE_PTR(k);
  S2MOE_REQUIRE_PTR(v);
  S2MOE_REQUIRE_INTS(tok_off);
  S2MOE_REQUIRE_PTR(out);
  const s2moe_attn& t = *attn;
  const int elt = t.dtype == S2MOE_F32 ? 4 : 2, D = t.head_dim;
  if ((st = check_rows(fn, "ldq", t.ldq, t.n_heads, D, elt)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldk", t.ldk, t.n_kv_heads, D, elt)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldv", t.ldv, t.n_kv_heads, D, elt)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldo", t.ldo, t.n_heads, D, elt)) != S2MOE_OK) return st;
  const int64_t wq = (int64_t)t.n_heads * D * elt, wk = (int64_t)t.n_kv_heads * D * elt;
  if (rows_meet(q, t.ldq * elt, wq, out, t.ldo * elt, wq, n_tokens) ||
      rows_meet(k, t.ldk * elt, wk, out, t.ldo * elt, wq, n_tokens) ||
      rows_meet(v, t.ldv * elt, wk, out, t.ldo * elt, wq, n_tokens))
    return fail(S2MOE_EINVAL, "%s: out overlaps q, k or v", fn);
  s2moe::PromptArgs a;
  a.Hq = t.n_heads;
  a.Hkv = t.n_kv_heads;
  a.G = t.n_heads / t.n_kv_heads;
  a.D = D;
  a.f32 = t.dtype == S2MOE_F32;
  a.n = n;
  a.n_tokens = n_tokens;
  a.tok_off = tok_off;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.out = static_cast<char*>(out);
  a.ldq = t.ldq;
  a.ldk = t.ldk;
  a.ldv = t.ldv;
  a.ldo = t.ldo;
  a.scale = t.scale;
  return hip_status(fn, s2moe::launch_prompt_attention(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
