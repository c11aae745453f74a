// Internal launch interface of the cache and attention kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace s2moe {

constexpr int kKvMaxRequests = 1024;  // S2MOE_KV_MAX_REQUESTS
constexpr int kMaxNodes = 256;        // nodes of a drafted tree (S2MOE_MAX_TOKENS)

enum : int32_t { kKvNoPages = 1, kKvTooLong = 2, kKvBadSeq = 4, kKvBusy = 8, kKvBadPath = 16 };

// The caller's cache (s2moe_kv_cache), with one layer's sizes worked out.
struct KvCache {
  int L, Hkv, D, n_pages, P, log_p, max_seqs, max_pages;
  bool f32;
  char* k;
  char* v;
  int32_t* table;
  int32_t* length;
  int32_t* refs;

  __host__ __device__ int elt() const { return f32 ? 4 : 2; }
  // Bytes of one head's part of a page, of a page and of a layer's pool.
  __host__ __device__ int64_t head_bytes() const { return (int64_t)P * D * elt(); }
  __host__ __device__ int64_t page_bytes() const { return head_bytes() * Hkv; }
  __host__ __device__ int64_t layer_bytes() const { return page_bytes() * n_pages; }
};

// Lets `kernel` have up to `bytes` of dynamic LDS on the current device; `done`, the
// kernel's own, has a bit for each device where that has been asked for.
inline hipError_t allow_lds(const void* kernel, size_t bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

hipError_t launch_kv_init(const KvCache& c, hipStream_t s);
hipError_t launch_kv_fork(const KvCache& c, int n, const int32_t* src, const int32_t* dst,
                          int32_t* status, hipStream_t s);
hipError_t launch_kv_reserve(const KvCache& c, int n, const int32_t* seqs, const int32_t* extra,
                             int32_t* copied, int32_t* status, hipStream_t s);
hipError_t launch_kv_commit(const KvCache& c, int n, int max_path, const int32_t* seqs,
                            const int32_t* path, const int32_t* n_accept, int32_t* status,
                            hipStream_t s);
hipError_t launch_kv_free(const KvCache& c, int n, const int32_t* seqs, int32_t* status,
                          hipStream_t s);

struct AppendArgs {
  int layer, n, n_tokens;
  const int32_t* seqs;
  const int32_t* tok_off;
  const char* k;
  const char* v;
  int64_t ldk, ldv;  // elements
};
hipError_t launch_kv_append(const KvCache& c, const AppendArgs& a, hipStream_t s);

// Without parents: each request's tokens one after another.
hipError_t launch_positions(const KvCache& c, int n, int n_tokens, const int32_t* seqs,
                            const int32_t* tok_off, const int32_t* parent, int32_t* pos,
                            hipStream_t s);

struct RotateArgs {
  int layer, n, n_tokens, Hq, rot;
  bool neighbours;  // pairs of coordinates 2 j and 2 j + 1, else j and j + rot / 2
  const int32_t* seqs;
  const int32_t* tok_off;
  const int32_t* pos;
  const float* freq;
  const char* q;
  const char* k;
  const char* v;
  char* q_out;
  char* k_out;  // or null
  int64_t ldq, ldk, ldv, ldqo, ldko;  // elements
};
hipError_t launch_append_rotated(const KvCache& c, const RotateArgs& a, hipStream_t s);

struct TreeArgs {
  const char* k;  // the layer's pools
  const char* v;
  const int32_t* table;
  const int32_t* length;
  int n_pages, P, log_p, max_seqs, max_pages;
  int Hq, Hkv, G, D;  // G = Hq / Hkv
  bool f32;
  int n, n_tokens, max_nodes;
  const int32_t* seqs;
  const int32_t* tok_off;
  const int32_t* parent;
  const char* q;
  char* out;
  int64_t ldq, ldo;  // elements
  float scale;
  float* ws;
};
// Of a's head counts, head size, type and max_nodes alone.
size_t tree_attention_workspace(const TreeArgs& a);
hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t s);

struct PromptArgs {
  int Hq, Hkv, G, D;
  bool f32;
  int n, n_tokens;
  const int32_t* tok_off;
  const char* q;
  const char* k;
  const char* v;
  char* out;
  int64_t ldq, ldk, ldv, ldo;  // elements
  float scale;
};
hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t s);

}  // namespace s2moe
