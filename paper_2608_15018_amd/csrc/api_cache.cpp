// C-ABI entry points of the cache and attention operators: argument checks
// on the host, then kernel launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "attention.h"
#include "rows.h"
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
using s2moe::bytes_meet;
using s2moe::check_rows;
using s2moe::fail;
using s2moe::hip_status;
using s2moe::ok;
using s2moe::rows_meet;

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

s2moe_status check_tokens(const char* fn, int32_t n_tokens) {
  if (n_tokens < 0) return fail(S2MOE_EINVAL, "%s: n_tokens = %d < 0", fn, n_tokens);
  if (n_tokens > 1 << 28)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_tokens = %d exceeds 2^28", fn, n_tokens);
  return S2MOE_OK;
}

// Whether `n` bytes at `p` meet one of the cache's arrays.
bool meets_cache(const s2moe::KvCache& c, const void* p, int64_t n) {
  const int64_t pool = c.L * c.layer_bytes();
  return bytes_meet(p, n, c.k, pool) || bytes_meet(p, n, c.v, pool) ||
         bytes_meet(p, n, c.table, (int64_t)c.max_seqs * c.max_pages * 4) ||
         bytes_meet(p, n, c.length, (int64_t)c.max_seqs * 4) ||
         bytes_meet(p, n, c.refs, (int64_t)c.n_pages * 4);
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

s2moe_status s2moe_kv_positions(const s2moe_kv_cache* cache, int32_t n, int32_t n_tokens,
                                const int32_t* seqs, const int32_t* tok_off, const int32_t* parent,
                                int32_t* pos, void* stream) {
  const char* fn = "s2moe_kv_positions";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st == S2MOE_OK) st = check_tokens(fn, n_tokens);
  if (st != S2MOE_OK) return st;
  if (n == 0 || n_tokens == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(tok_off);
  S2MOE_REQUIRE_INTS(pos);
  if (parent != nullptr && !aligned(parent, 4))
    return fail(S2MOE_EINVAL, "%s: parent is not 4-byte aligned", fn);
  const int64_t bytes = (int64_t)n_tokens * 4;
  if (bytes_meet(pos, bytes, seqs, (int64_t)n * 4) ||
      bytes_meet(pos, bytes, tok_off, ((int64_t)n + 1) * 4) ||
      (parent != nullptr && bytes_meet(pos, bytes, parent, bytes)))
    return fail(S2MOE_EINVAL, "%s: pos overlaps seqs, tok_off or parent", fn);
  if (meets_cache(c, pos, bytes))
    return fail(S2MOE_EINVAL, "%s: pos overlaps an array of the cache", fn);
  return hip_status(fn, s2moe::launch_positions(c, n, n_tokens, seqs, tok_off, parent, pos,
                                                static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_kv_append_rotated(const s2moe_kv_cache* cache, int32_t layer,
                                     const s2moe_rotation* rotation, int32_t n, int32_t n_tokens,
                                     const int32_t* seqs, const int32_t* tok_off,
                                     const int32_t* pos, const float* inv_freq, const void* q,
                                     const void* k, const void* v, void* q_out, void* k_out,
                                     void* stream) {
  const char* fn = "s2moe_kv_append_rotated";
  s2moe::KvCache c;
  s2moe_status st = check_cache(fn, cache, &c);
  if (st == S2MOE_OK) st = check_requests(fn, n);
  if (st == S2MOE_OK) st = check_layer_index(fn, c, layer);
  if (st == S2MOE_OK) st = check_tokens(fn, n_tokens);
  if (st != S2MOE_OK) return st;
  if (rotation == nullptr) return fail(S2MOE_EINVAL, "%s: rotation is NULL", fn);
  const s2moe_rotation& r = *rotation;
  if (r.n_heads < 1) return fail(S2MOE_EINVAL, "%s: n_heads = %d < 1", fn, r.n_heads);
  if (r.n_heads > 1024)
    return fail(S2MOE_EUNSUPPORTED, "%s: n_heads = %d exceeds 1024", fn, r.n_heads);
  if (r.rot_dim < 16 || r.rot_dim > c.D || r.rot_dim % 16 != 0)
    return fail(S2MOE_EINVAL, "%s: rot_dim = %d must be a multiple of 16 in [16, %d]", fn,
                r.rot_dim, c.D);
  if (r.neighbours != 0 && r.neighbours != 1)
    return fail(S2MOE_EINVAL, "%s: neighbours = %d must be 0 or 1", fn, r.neighbours);
  if ((int64_t)n_tokens * (c.Hkv + 40) > (int64_t)1 << 30)  // threads of a launch, below 2^32
    return fail(S2MOE_EUNSUPPORTED, "%s: n_tokens (n_kv_heads + 40) = %d %d exceeds 2^30", fn,
                n_tokens, c.Hkv + 40);
  if (n == 0 || n_tokens == 0) return ok();
  S2MOE_REQUIRE_INTS(seqs);
  S2MOE_REQUIRE_INTS(tok_off);
  S2MOE_REQUIRE_INTS(pos);
  S2MOE_REQUIRE_INTS(inv_freq);
  S2MOE_REQUIRE_PTR(q);
  S2MOE_REQUIRE_PTR(k);
  S2MOE_REQUIRE_PTR(v);
  S2MOE_REQUIRE_PTR(q_out);
  if (k_out != nullptr && !aligned16(k_out))
    return fail(S2MOE_EINVAL, "%s: k_out is not 16-byte aligned", fn);
  const int e = c.elt();
  if ((st = check_rows(fn, "ldq", r.ldq, r.n_heads, c.D, e)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldk", r.ldk, c.Hkv, c.D, e)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldv", r.ldv, c.Hkv, c.D, e)) != S2MOE_OK) return st;
  if ((st = check_rows(fn, "ldqo", r.ldqo, r.n_heads, c.D, e)) != S2MOE_OK) return st;
  if (k_out != nullptr && (st = check_rows(fn, "ldko", r.ldko, c.Hkv, c.D, e)) != S2MOE_OK)
    return st;
  const int64_t wq = (int64_t)r.n_heads * c.D * e, wk = (int64_t)c.Hkv * c.D * e;
  const int64_t lq = r.ldq * e, lk = r.ldk * e, lv = r.ldv * e, lqo = r.ldqo * e, lko = r.ldko * e;
  // In place: each element is read and written by one lane.
  const bool same_q = q_out == q && lqo == lq, same_k = k_out == k && lko == lk;
  if ((!same_q && rows_meet(q_out, lqo, wq, q, lq, wq, n_tokens)) ||
      rows_meet(q_out, lqo, wq, k, lk, wk, n_tokens) ||
      rows_meet(q_out, lqo, wq, v, lv, wk, n_tokens))
    return fail(S2MOE_EINVAL, "%s: q_out overlaps q (other than in place), k or v", fn);
  if (k_out != nullptr && ((!same_k && rows_meet(k_out, lko, wk, k, lk, wk, n_tokens)) ||
                           rows_meet(k_out, lko, wk, q, lq, wq, n_tokens) ||
                           rows_meet(k_out, lko, wk, v, lv, wk, n_tokens) ||
                           rows_meet(k_out, lko, wk, q_out, lqo, wq, n_tokens)))
    return fail(S2MOE_EINVAL, "%s: k_out overlaps k (other than in place), q, v or q_out", fn);
  const auto meets_ints = [&](const void* out, int64_t ld, int64_t width) {
    const int64_t bytes = (n_tokens - 1) * ld + width;
    return bytes_meet(out, bytes, pos, (int64_t)n_tokens * 4) ||
           bytes_meet(out, bytes, inv_freq, (int64_t)r.rot_dim * 2) ||
           bytes_meet(out, bytes, seqs, (int64_t)n * 4) ||
           bytes_meet(out, bytes, tok_off, ((int64_t)n + 1) * 4);
  };
  if (meets_ints(q_out, lqo, wq) || (k_out != nullptr && meets_ints(k_out, lko, wk)))
    return fail(S2MOE_EINVAL, "%s: q_out or k_out overlaps pos, inv_freq, seqs or tok_off", fn);
  if (meets_cache(c, q_out, (n_tokens - 1) * lqo + wq) ||
      (k_out != nullptr && meets_cache(c, k_out, (n_tokens - 1) * lko + wk)))
    return fail(S2MOE_EINVAL, "%s: q_out or k_out overlaps an array of the cache", fn);
  s2moe::RotateArgs a;
  a.layer = layer;
  a.n = n;
  a.n_tokens = n_tokens;
  a.Hq = r.n_heads;
  a.rot = r.rot_dim;
  a.neighbours = r.neighbours != 0;
  a.seqs = seqs;
  a.tok_off = tok_off;
  a.pos = pos;
  a.freq = inv_freq;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.q_out = static_cast<char*>(q_out);
  a.k_out = static_cast<char*>(k_out);
  a.ldq = r.ldq;
  a.ldk = r.ldk;
  a.ldv = r.ldv;
  a.ldqo = r.ldqo;
  a.ldko = r.ldko;
  return hip_status(fn, s2moe::launch_append_rotated(c, a, static_cast<hipStream_t>(stream)));
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
