// Causal attention of packed prompts: one wave per (token, query head).
#include "attention.h"
#include "common.h"

namespace s2moe {
namespace {

__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ float load(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store(float* p, float x) { *p = x; }
__device__ __forceinline__ void store(uint16_t* p, float x) { *p = (uint16_t)f32_to_bf16(x); }

template <typename E, int D>
__global__ __launch_bounds__(64) void prompt_kernel(PromptArgs a) {
  __shared__ float q_s[D], p_s[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.tok_off[mid] <= t) lo = mid; else hi = mid;
  }
  const int first = a.tok_off[lo];
  if (first < 0 || t < first || t >= a.tok_off[lo + 1]) return;
  const E* q = reinterpret_cast<const E*>(a.q) + t * a.ldq + h * D;
  for (int d = lane; d < D; d += 64) q_s[d] = load(q + d);
  __syncthreads();
  const int total = t - first + 1, g = h / a.G;
  float m = -INFINITY, l = 0.f, acc[D / 64];
  for (int i = 0; i < D / 64; ++i) acc[i] = 0.f;
  for (int k0 = 0; k0 < total; k0 += 64) {
    const int key = k0 + lane;
    const bool vis = key < total;
    float x = -INFINITY;
    if (vis) {
      const E* kp = reinterpret_cast<const E*>(a.k) + (first + key) * a.ldk + g * D;
      x = 0.f;
      for (int d = 0; d < D; ++d) x = fmaf(q_s[d], load(kp + d), x);
      x *= a.scale;
    }
    float top = x;
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float m2 = fmaxf(m, top);
    const float keep = expf(m - m2), p = vis ? expf(x - m2) : 0.f;
    float sum = p;
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    l = l * keep + sum;
    m = m2;
    for (int i = 0; i < D / 64; ++i) acc[i] *= keep;
    p_s[lane] = p;
    __syncthreads();
    const int n = total - k0 < 64 ? total - k0 : 64;
    for (int j = 0; j < n; ++j) {
      const E* vp = reinterpret_cast<const E*>(a.v) + (first + k0 + j) * a.ldv + g * D;
      for (int i = 0; i < D / 64; ++i) acc[i] = fmaf(p_s[j], load(vp + lane + 64 * i), acc[i]);
    }
    __syncthreads();
  }
  E* o = reinterpret_cast<E*>(a.out) + t * a.ldo + h * D;
  for (int i = 0; i < D / 64; ++i) store(o + lane + 64 * i, acc[i] / l);
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t s) {
  const dim3 grid(a.n_tokens, a.Hq);
  if (a.f32) {
    if (a.D == 64) prompt_kernel<float, 64><<<grid, 64, 0, s>>>(a);
    else prompt_kernel<float, 128><<<grid, 64, 0, s>>>(a);
  } else {
    if (a.D == 64) prompt_kernel<uint16_t, 64><<<grid, 64, 0, s>>>(a);
    else prompt_kernel<uint16_t, 128><<<grid, 64, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace s2moe
