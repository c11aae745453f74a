// Products of 8-bit rows and weights with a scale for each block of 128:
//
//   y[i][j] = sum over blocks b of xs[b][i] ws[j / 128][b] (sum over k in b of x[i][k] w[j][k])
//
// One matrix instruction takes a whole block: 16 weight rows by 16 tokens by 128, in
// fp32.  Its four results a lane belong to one token and to weight rows of one scale, so
// the block's two scales are one factor a lane, and adding the block to the sum is one
// fused multiply-add a result.  Both operands name k alike, so that a lane may hold any
// 32 of a block's elements: here two pieces of 16 bytes, 64 bytes apart, as rows lie.
//
// The 8-bit instruction adds eight neighbouring products after cutting each off 13 bits
// below the largest one's exponent, towards zero (measured; the eights then add up in
// fp32): of normal data 1.4e-5 of the result, a hundredth of bf16's rounding and so left
// to it.  Results in fp32 come from the 16-bit instruction on the same codes, which fp16
// holds exactly and whose products it adds in fp32 (measured: 1e-8 on the same data); it
// does half as much in the same time.
#include "attn_common.h"
#include "dense.h"

namespace s2moe {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;

typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;

__device__ __forceinline__ f16x8 to_f16(int lo, int hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The products of a block; kWide: for results in fp32.
template <bool kWide>
__device__ __forceinline__ f32x4 mma(i32x8 w, i32x8 x) {
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if constexpr (kWide) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_f16(w[2 * i], w[2 * i + 1]), to_f16(x[2 * i], x[2 * i + 1]), y, 0, 0, 0);
    return y;
  }
  // Scale operands of zero with the formats 0, 0 (e4m3): the product without scales.
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, y, 0, 0, 0, 0, 0, 0);
}

// A lane's 32 elements of block b of a row, zeros past k.
__device__ __forceinline__ i32x8 load_block(const uint8_t* row, int k0, int k, int quarter) {
  u32x4 p[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = k0 + 64 * i + 16 * quarter;
    p[i] = at < k ? *reinterpret_cast<const u32x4*>(row + at) : u32x4{0, 0, 0, 0};
  }
  return i32x8{(int)p[0][0], (int)p[0][1], (int)p[0][2], (int)p[0][3], (int)p[1][0], (int)p[1][1], (int)p[1][2], (int)p[1][3]};
}

// Four neighbouring results of a token; `vec`: all are inside and the row's start allows
// one store.
template <bool kF32Out>
__device__ __forceinline__ void store4(char* row, int col, int n, bool vec, f32x4 y) {
  if constexpr (kF32Out) {
    float* p = reinterpret_cast<float*>(row) + col;
    if (vec) {
      *reinterpret_cast<f32x4*>(p) = y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < n) p[i] = y[i];
    }
  } else {
    __bf16* p = reinterpret_cast<__bf16*>(row) + col;
    const bf16x2 lo = pack2(y[0], y[1]), hi = pack2(y[2], y[3]);
    if (vec) {
      *reinterpret_cast<bf16x4*>(p) = bf16x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < n) p[i] = i < 2 ? lo[i] : hi[i - 2];
    }
  }
}

// Few tokens: the weights' way from memory is what takes time.  A workgroup has 16 weight
// rows and 16 kTokens tokens; its waves take the blocks of k in turn, so that together
// they read stretches of the rows, and their sums are added in the waves' order.
template <int kTokens, int kWaves, bool kF32Out>
__global__ __launch_bounds__(kWaves * 64) void few_tokens_kernel(MatmulArgs a) {
  __shared__ f32x4 part[kWaves][kTokens][64];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, at = lane & 15;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * kTokens;
  const uint8_t* w = a.w + min(n0 + at, a.n - 1) * a.ldw;
  const float* ws = a.ws + (n0 / kBlock) * a.ldws;
  const uint8_t* x[kTokens];
  int token[kTokens];
#pragma unroll
  for (int t = 0; t < kTokens; ++t) {
    token[t] = min(m0 + 16 * t + at, a.m - 1);
    x[t] = a.x + token[t] * a.ldx;
  }
  f32x4 sum[kTokens] = {};
  for (int k0 = wave * kBlock; k0 < a.k; k0 += kWaves * kBlock) {
    const int b = k0 / kBlock;
    const i32x8 wb = load_block(w, k0, a.k, quarter);
    i32x8 xb[kTokens];
    float f[kTokens];
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      xb[t] = load_block(x[t], k0, a.k, quarter);
      f[t] = a.xs[b * a.ldxs + token[t]];
    }
    const float g = ws[b];
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      const f32x4 y = mma<kF32Out>(wb, xb[t]);
      const float scale = f[t] * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[t][i] = fmaf(y[i], scale, sum[t][i]);
    }
  }
#pragma unroll
  for (int t = 0; t < kTokens; ++t) part[wave][t][lane] = sum[t];
  __syncthreads();
  const int elt = kF32Out ? 4 : 2, col = n0 + 4 * quarter;
  const bool vec = col + 4 <= a.n && (a.ldo * elt & (4 * elt - 1)) == 0;
  for (int t = wave; t < kTokens; t += kWaves) {
    f32x4 y = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) y += part[v][t][lane];
    const int to = m0 + 16 * t + at;
    if (to < a.m && col < a.n) store4<kF32Out>(a.out + to * a.ldo * elt, col, a.n, vec, y);
  }
}

template <int kTokens, int kWaves>
void launch_few(const MatmulArgs& a, hipStream_t s) {
  const dim3 grid((a.n + 15) / 16, (a.m + 16 * kTokens - 1) / (16 * kTokens));
  if (a.f32) few_tokens_kernel<kTokens, kWaves, true><<<grid, kWaves * 64, 0, s>>>(a);
  else few_tokens_kernel<kTokens, kWaves, false><<<grid, kWaves * 64, 0, s>>>(a);
}

}  // namespace

hipError_t launch_scaled_matmul(const MatmulArgs& a, hipStream_t s) {
  if (a.m <= 16) launch_few<1, 8>(a, s);
  else launch_few<4, 8>(a, s);
  return hipGetLastError();
}

}  // namespace s2moe
