// Attention of drafted tokens over the cache: one wave per (node, query head).
#include "attention.h"
#include "common.h"

namespace s2moe {
namespace {

__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ float load(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store(float* p, float x) { *p = x; }
__device__ __forceinline__ void store(uint16_t* p, float x) { *p = (uint16_t)f32_to_bf16(x); }

template <typename E, int D>
__global__ __launch_bounds__(64) void tree_kernel(TreeArgs a) {
  __shared__ float q_s[D], p_s[64];
  __shared__ uint32_t seen_s[kMaxNodes / 32];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.tok_off[mid] <= t) lo = mid; else hi = mid;
  }
  const int first = a.tok_off[lo];
  int T = a.tok_off[lo + 1] - first;
  const int s = a.seqs[lo], node = t - first;
  if (first < 0 || node < 0 || node >= T || node >= a.max_nodes || s < 0 || s >= a.max_seqs) return;
  T = T < a.max_nodes ? T : a.max_nodes;
  if (lane < kMaxNodes / 32) seen_s[lane] = 0;
  const E* q = reinterpret_cast<const E*>(a.q) + t * a.ldq + h * D;
  for (int d = lane; d < D; d += 64) q_s[d] = load(q + d);
  __syncthreads();
  bool ok = true;
  if (lane == 0) {
    int j = node;
    for (;;) {
      seen_s[j >> 5] |= 1u << (j & 31);
      const int p = a.parent[first + j];
      if (p == -1) break;
      if (p < 0 || p >= j) { ok = false; break; }
      j = p;
    }
  }
  ok = __shfl(ok, 0);
  __syncthreads();
  const int len = a.length[s], cap = a.max_pages << a.log_p;
  int total = len + T;
  total = total < cap ? total : cap;
  if (!ok) total = 0;
  const int g = h / a.G;
  const int64_t page_elems = (int64_t)a.Hkv * a.P * D;
  const int32_t* row = a.table + (int64_t)s * a.max_pages;
  float m = -INFINITY, l = 0.f, acc[D / 64];
  for (int i = 0; i < D / 64; ++i) acc[i] = 0.f;
  for (int k0 = 0; k0 < total; k0 += 64) {
    const int key = k0 + lane;
    bool vis = key < total;
    if (vis && key >= len) vis = (seen_s[(key - len) >> 5] >> ((key - len) & 31)) & 1;
    float x = -INFINITY;
    if (vis) {
      int page = row[key >> a.log_p];
      page = page < 0 ? 0 : (page >= a.n_pages ? a.n_pages - 1 : page);
      const E* kp = reinterpret_cast<const E*>(a.k) + page * page_elems +
                    ((int64_t)g * a.P + (key & (a.P - 1))) * D;
      x = 0.f;
      for (int d = 0; d < D; ++d) x = fmaf(q_s[d], load(kp + d), x);
      x *= a.scale;
    }
    float top = x;
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float m2 = fmaxf(m, top);
    const float shift = m2 == -INFINITY ? 0.f : m2;
    const float keep = expf(m - shift), p = vis ? expf(x - shift) : 0.f;
    float sum = p;
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    l = l * keep + sum;
    m = m2;
    for (int i = 0; i < D / 64; ++i) acc[i] *= keep;
    p_s[lane] = p;
    uint64_t mask = __ballot(vis);
    __syncthreads();
    for (; mask != 0; mask &= mask - 1) {
      const int j = __ffsll((unsigned long long)mask) - 1, kk = k0 + j, slot = kk & (a.P - 1);
      int page = row[kk >> a.log_p];
      page = page < 0 ? 0 : (page >= a.n_pages ? a.n_pages - 1 : page);
      const E* vp = reinterpret_cast<const E*>(a.v) + page * page_elems + (int64_t)g * a.P * D +
                    (slot >> 3) * D * 8 + (slot & 7);
      for (int i = 0; i < D / 64; ++i) acc[i] = fmaf(p_s[j], load(vp + (lane + 64 * i) * 8), acc[i]);
    }
    __syncthreads();
  }
  E* o = reinterpret_cast<E*>(a.out) + t * a.ldo + h * D;
  for (int i = 0; i < D / 64; ++i) store(o + lane + 64 * i, l == 0.f ? 0.f : acc[i] / l);
}

}  // namespace

size_t tree_attention_workspace(int, int, int, bool, int, int) { return 256; }

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t s) {
  const dim3 grid(a.n_tokens, a.Hq);
  if (a.f32) {
    if (a.D == 64) tree_kernel<float, 64><<<grid, 64, 0, s>>>(a);
    else tree_kernel<float, 128><<<grid, 64, 0, s>>>(a);
  } else {
    if (a.D == 64) tree_kernel<uint16_t, 64><<<grid, 64, 0, s>>>(a);
    else tree_kernel<uint16_t, 128><<<grid, 64, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace s2moe
