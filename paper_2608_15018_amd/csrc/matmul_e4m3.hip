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
// fp32): of normal data 1.4e-5 of the result (2-norm), a hundredth of bf16's rounding and so
// left to it.  No more than 2^-10 of the sum of the products' magnitudes, as the largest is
// not cut: seven lose less than 2^-13 of it each (2^-7 where a code below 2^-6, whose exponent
// counts as -6, makes the largest).  Results in fp32 come from the 16-bit instruction on the
// same codes, which fp16 holds exactly and whose products it adds in fp32 (measured on the
// same data: results of one block off by 3.7e-8, of which 2.6e-8 is their own rounding, of 32
// blocks by 7e-8 to 1.1e-7); it does half as much in the same time.
#include <atomic>
#include <cmath>
#include <type_traits>

#include "attention.h"
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

__device__ __forceinline__ i32x8 join(u32x4 p, u32x4 q) {
  return i32x8{(int)p[0], (int)p[1], (int)p[2], (int)p[3], (int)q[0], (int)q[1], (int)q[2], (int)q[3]};
}
// A lane's elements of the last block, `rest` long: zeros past its end.
__device__ __forceinline__ i32x8 cut_off(i32x8 v, int quarter, int rest) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 16 * quarter + 64 * (i / 4) < rest ? v[i] : 0;
  return v;
}

// Loads to LDS as in load_to_lds, of which the LDS address is a number already.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load16(const char* base, uint32_t off, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(off), "s"(base) : "memory", "m0");
}
// The same of weights, kOnce: that no other workgroup reads, which leaves the caches to the
// rest (16 x 32000 x 4096: 24.5 us, 27.3 without; weights that several read take longer so).
template <bool kOnce>
__device__ __forceinline__ void load16_w(const char* base, uint32_t off, uint32_t at) {
  if constexpr (kOnce)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(at), "v"(off), "s"(base) : "memory", "m0");
  else
    load16(base, off, at);
}
__device__ __forceinline__ void load4(const char* base, uint32_t off, uint32_t at) {  // 256 bytes a wave
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(at), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const char* lds) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds);
}
// Of the waves alone: who reads what another has loaded waits for loads before it.
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" : : : "memory"); }
// The load of x is waited for here and not at its first use, where the compiler, which
// does not know of the loads to LDS, would wait for all of those too.
__device__ __forceinline__ void arrived(float& x) { asm volatile("" : "+v"(x)); }

// The workgroup's tile: each of the eight dies takes a stretch of the tiles, in strips four
// tiles of weights wide, so that its second-level cache holds what its workgroups share
// (8193 x 6144 x 4096 with strips of one, two, four, eight: 191, 178, 175, 175 us; 251 x 5120
// x 2880, from memory: 13.7, 13.6, 13.3, 14.5).
constexpr int kStrip = 4;
__device__ __forceinline__ bool tile_of(int tiles_n, int tiles_m, int* tn, int* tm) {
  const int tiles = tiles_n * tiles_m, per = (tiles + 7) / 8;
  const int nth = blockIdx.x >> 3, tile = (blockIdx.x & 7) * per + nth;
  if (nth >= per || tile >= tiles) return false;
  const int strip = tile / (kStrip * tiles_m), in = tile - strip * kStrip * tiles_m, wide = min(kStrip, tiles_n - strip * kStrip);
  *tn = strip * kStrip + in % wide;
  *tm = in / wide;
  return true;
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

template <int TN, int TM, bool kF32Out>
__device__ __forceinline__ void store_tile(const MatmulArgs& a, int my_n, int my_m, int quarter, int at, const f32x4 (&sum)[TN][TM]) {
  constexpr int elt = kF32Out ? 4 : 2;
  const bool even = (a.ldo * elt & (4 * elt - 1)) == 0;
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int to = my_m + 16 * t + at;
    if (to >= a.m) continue;
    char* const row = a.out + to * a.ldo * elt;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const int col = my_n + 16 * i + 4 * quarter;
      if (col < a.n) store4<kF32Out>(row, col, a.n, even && col + 4 <= a.n, sum[i][t]);
    }
  }
}

// The same by way of LDS, a stretch of whole rows at a time: results lie 32 bytes of a row to
// 16 rows in the lanes, and stored so they would take 32 us of 202 at 8192 x 6144 x 4096.
// Past the caches, which the operands need: 175 us there instead of 183.
// `scratch`: the wave's own kScratch<..> bytes, which nothing else uses any more.
template <int TN, int TM, bool kF32Out>
constexpr int kScratch = 16 * TM * (16 * TN * (kF32Out ? 4 : 2) + 16);
template <int TN, int TM, bool kF32Out>
__device__ __forceinline__ void store_rows(const MatmulArgs& a, int my_n, int my_m, int quarter, int at, const f32x4 (&sum)[TN][TM],
                                           char* scratch) {
  constexpr int elt = kF32Out ? 4 : 2, kRow = 16 * TN * elt, kStep = kRow + 16, kPieces = kRow / 16, kAtOnce = 64 / kPieces;
  if (kAtOnce > 16 * TM || a.ldo * elt % 16 != 0 || my_n + 16 * TN > a.n) {
    store_tile<TN, TM, kF32Out>(a, my_n, my_m, quarter, at, sum);
    return;
  }
#pragma unroll
  for (int t = 0; t < TM; ++t)
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      char* const p = scratch + (16 * t + at) * kStep + (16 * i + 4 * quarter) * elt;
      if constexpr (kF32Out) {
        *reinterpret_cast<f32x4*>(p) = sum[i][t];
      } else {
        const bf16x2 lo = pack2(sum[i][t][0], sum[i][t][1]), hi = pack2(sum[i][t][2], sum[i][t][3]);
        *reinterpret_cast<bf16x4*>(p) = bf16x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int lane = 16 * quarter + at, piece = lane % kPieces;
#pragma unroll
  for (int r0 = 0; r0 < 16 * TM; r0 += kAtOnce) {
    const int r = r0 + lane / kPieces, to = my_m + r;
    const u32x4 v = *reinterpret_cast<const u32x4*>(scratch + r * kStep + piece * 16);
    if (to < a.m) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a.out + (to * a.ldo + my_n) * elt + piece * 16));
  }
}

// Up to 32 tokens a tile: how soon the weights come is what takes time, their latency or,
// of many, their bytes (16 x 32000 x 4096: 24.7 us, 5.3 TB/s of weights).  A workgroup has
// 16 TN weight rows and 16 TM tokens; its waves take the blocks of k in turn, kAhead of them
// on their way to LDS at any time, each to the wave's own places, so that no wave waits for
// another before the sums are added, in the waves' order.  Eight lanes read 128 bytes of a
// row, four times the lines a load that the operands' layout would have (16 x 6144 x 4096:
// 7.2 us, 9.2 with loads straight to registers).  Workgroups begin at different blocks: rows
// that lie 4096 bytes apart, read in step, would come from few of the memory's channels.
template <int TN, int TM, int kAhead, int kWaves, bool kF32Out, bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void stream_kernel(MatmulArgs a, int tiles_n, int tiles_m) {
  constexpr int kRows = 16 * (TN + TM), kLoads = 2 * (TN + TM) + 1, kStage = kRows * kBlock + 256;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, at = lane & 15;
  int tn, tm;
  if (!tile_of(tiles_n, tiles_m, &tn, &tm)) return;
  const int n0 = tn * 16 * TN, m0 = tm * 16 * TM;
  const int steps = (a.k + kBlock - 1) / kBlock, rest = a.k - (steps - 1) * kBlock;
  const int piece = (lane & 7) ^ (lane >> 3);
  uint32_t woff[2 * TN], xoff[2 * TM];
#pragma unroll
  for (int i = 0; i < 2 * TN; ++i) woff[i] = (uint32_t)min(8 * i + (lane >> 3), a.n - 1 - n0) * (uint32_t)a.ldw + piece * 16;
#pragma unroll
  for (int i = 0; i < 2 * TM; ++i) xoff[i] = (uint32_t)min(8 * i + (lane >> 3), a.m - 1 - m0) * (uint32_t)a.ldx + piece * 16;
  const uint32_t mine = 4u * min(m0 + (lane & (16 * TM - 1)), a.m - 1);
  const char* const wbase = reinterpret_cast<const char*>(a.w) + n0 * a.ldw;
  const char* const xbase = reinterpret_cast<const char*>(a.x) + m0 * a.ldx;
  const float* const ws = a.ws + n0 / kBlock * a.ldws;
  const int count = wave < steps ? (steps - 1 - wave) / kWaves + 1 : 0;
  const int turn = count > 0 ? tn % count : 0;
  const auto block_of = [&](int i) {
    int j = i + turn;
    if (j >= count) j -= count;
    return wave + j * kWaves;
  };
  char* const mylds = lds + wave * kAhead * kStage;
  const uint32_t at0 = lds_address(mylds);
  float wscale = 0.f;
  // Block i of the wave's; past its last the last one again.
  const auto load = [&](int i, int slot) {
    const int b = block_of(min(i, count - 1));
    const uint32_t st = at0 + slot * kStage;
    const uint32_t back = b == steps - 1 && piece * 16 >= rest ? (uint32_t)(piece * 16 - rest + 16) : 0u;
#pragma unroll
    for (int l = 0; l < 2 * TN; ++l) load16_w<kOnce>(wbase + b * kBlock, woff[l] - back, st + l * 1024);
#pragma unroll
    for (int l = 0; l < 2 * TM; ++l) load16(xbase + b * kBlock, xoff[l] - back, st + (2 * TN + l) * 1024);
    load4(reinterpret_cast<const char*>(a.xs + b * a.ldxs), mine, st + kRows * kBlock);
  };
  const int lo = at * kBlock + ((quarter ^ (at & 7)) * 16), hi = lo ^ 64;
  f32x4 sum[TN][TM] = {};
  if (count > 0) {
    wscale = ws[block_of(min(lane, count - 1))];
    arrived(wscale);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(i, i);
    int slot = 0;
    for (int i = 0; i < count; ++i) {
      if ((i & 63) == 0 && i > 0) {
        wscale = ws[block_of(min(i + lane, count - 1))];
        arrived(wscale);
      }
      wait_loads<(kAhead - 1) * kLoads>();
      const int b = block_of(i);
      const char* const stage = mylds + slot * kStage;
      const bool last = b == steps - 1 && rest < kBlock;
      const auto operand = [&](int row) {
        const char* const p = stage + row * kBlock;
        return join(*reinterpret_cast<const u32x4*>(p + lo), *reinterpret_cast<const u32x4*>(p + hi));
      };
      i32x8 wb[TN], xb[TM];
      float f[TM];
      const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscale), i & 63));
#pragma unroll
      for (int t = 0; t < TM; ++t) {
        xb[t] = operand(16 * (TN + t));
        f[t] = reinterpret_cast<const float*>(stage + kRows * kBlock)[16 * t + at] * g;
      }
#pragma unroll
      for (int n = 0; n < TN; ++n) wb[n] = operand(16 * n);
      wait_lds();  // this block's place takes a later one
      load(i + kAhead, slot);
      slot = slot == kAhead - 1 ? 0 : slot + 1;
      if (last) {
#pragma unroll
        for (int n = 0; n < TN; ++n) wb[n] = cut_off(wb[n], quarter, rest);
#pragma unroll
        for (int t = 0; t < TM; ++t) xb[t] = cut_off(xb[t], quarter, rest);
      }
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int t = 0; t < TM; ++t) {
          const f32x4 y = mma<kF32Out>(wb[n], xb[t]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[n][t][e] = fmaf(y[e], f[t], sum[n][t][e]);
        }
    }
    wait_loads<0>();
  }
  __syncthreads();  // the blocks' places become the sums'
  f32x4* const part = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int t = 0; t < TM; ++t) part[(wave * TN * TM + n * TM + t) * 64 + lane] = sum[n][t];
  __syncthreads();
#pragma unroll
  for (int q0 = 0; q0 < TN * TM; q0 += kWaves) {
    const int q = q0 + wave, n = q / TM, t = q % TM;
    if (q >= TN * TM) break;
    f32x4 y[1][1] = {{part[q * 64 + lane]}};
#pragma unroll
    for (int v = 1; v < kWaves; ++v) y[0][0] += part[(v * TN * TM + q) * 64 + lane];
    store_tile<1, 1, kF32Out>(a, n0 + 16 * n, m0 + 16 * t, quarter, at, y);
  }
}

// Up to 16 tokens a tile and several rounds of workgroups: as above, but straight into
// registers, for which a workgroup has nothing to set up (16 x 16384 x 2048: 9.1 us, 9.5 to
// 9.9 by way of LDS).
template <int TN, bool kF32Out>
__global__ __launch_bounds__(512) void few_tokens_kernel(MatmulArgs a, int tiles_n, int tiles_m) {
  constexpr int kWaves = 8;
  __shared__ f32x4 part[kWaves][TN][64];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, at = lane & 15;
  int tn, tm;
  if (!tile_of(tiles_n, tiles_m, &tn, &tm)) return;
  const int n0 = tn * 16 * TN, m0 = tm * 16;
  const int steps = (a.k + kBlock - 1) / kBlock, rest = a.k - (steps - 1) * kBlock;
  const char* const wbase = reinterpret_cast<const char*>(a.w) + n0 * a.ldw;
  const char* const xbase = reinterpret_cast<const char*>(a.x) + m0 * a.ldx;
  uint32_t woff[TN];  // rows past the last are read as the last
#pragma unroll
  for (int i = 0; i < TN; ++i) woff[i] = (uint32_t)min(16 * i + at, a.n - 1 - n0) * (uint32_t)a.ldw + 16 * quarter;
  const uint32_t token = min(at, a.m - 1 - m0), xoff = token * (uint32_t)a.ldx + 16 * quarter;
  const float* const ws = a.ws + n0 / kBlock * a.ldws;
  f32x4 sum[TN] = {};
  const int count = wave < steps ? (steps - 1 - wave) / kWaves + 1 : 0;  // this wave's blocks
  int j = count > 0 ? tn % count : 0;
  for (int c = 0; c < count; ++c) {
    const int b = wave + j * kWaves;
    j = j + 1 == count ? 0 : j + 1;
    // In the last block pieces past k are read as its last one, and not used.
    const bool last = b == steps - 1 && rest < kBlock;
    const uint32_t back = 16 * quarter - rest + 16;
    const uint32_t lo = last && 16 * quarter >= rest ? back : 0u, hi = last && 64 + 16 * quarter >= rest ? back : (uint32_t)-64;
    const char* const w = wbase + b * kBlock;
    const char* const x = xbase + b * kBlock;
    i32x8 wb[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i)
      wb[i] = join(*reinterpret_cast<const u32x4*>(w + (woff[i] - lo)), *reinterpret_cast<const u32x4*>(w + (woff[i] - hi)));
    i32x8 xb = join(*reinterpret_cast<const u32x4*>(x + (xoff - lo)), *reinterpret_cast<const u32x4*>(x + (xoff - hi)));
    const float f = (a.xs + b * a.ldxs + m0)[token] * ws[b];
    if (last) {
#pragma unroll
      for (int i = 0; i < TN; ++i) wb[i] = cut_off(wb[i], quarter, rest);
      xb = cut_off(xb, quarter, rest);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const f32x4 y = mma<kF32Out>(wb[i], xb);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[i][e] = fmaf(y[e], f, sum[i][e]);
    }
  }
#pragma unroll
  for (int i = 0; i < TN; ++i) part[wave][i][lane] = sum[i];
  __syncthreads();
  if (wave >= TN) return;
  f32x4 y[1][1] = {{part[0][wave][lane]}};
#pragma unroll
  for (int v = 1; v < kWaves; ++v) y[0][0] += part[v][wave][lane];
  store_tile<1, 1, kF32Out>(a, n0 + 16 * wave, m0, quarter, at, y);
}

// Tiles between: what a step costs beside its products is what takes time.  kStages blocks
// of k are in LDS or on their way there; while the matrix cores have one block's operands,
// the waves read the next one's.  Scales of tokens come the same way, 64 words a wave.
// How far ahead loads have to be, and how many workgroups a compute unit holds, decides: of
// 64 x 64 tiles one a unit takes 12.6 us at 128 x 5120 x 2880 with four blocks, 13.7 with
// three, two a unit 18.8 and 18.2 at 384; 64 x 96 tiles, three blocks, keep 251 tokens to
// one a unit: 14.8 us, 18.2 with 64 x 64.
template <int WN, int WM, int TN, int TM, int kStages, bool kF32Out, bool kOnce>
__global__ __launch_bounds__(64 * WN * WM) void small_tiles_kernel(MatmulArgs a, int tiles_n, int tiles_m) {
  constexpr int kN = 16 * TN * WN, kM = 16 * TM * WM, kWaves = WN * WM;
  constexpr int kLoadsW = kN / 8 / kWaves, kLoadsX = kM / 8 / kWaves, kLoads = kLoadsW + kLoadsX + 1;
  static_assert(kN % (8 * kWaves) == 0 && kM % (8 * kWaves) == 0 && 16 * TN <= kBlock, "rows");
  constexpr int kStage = (kN + kM) * kBlock + kWaves * 256;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, at = lane & 15;
  int n0, m0;
  if (!tile_of(tiles_n, tiles_m, &n0, &m0)) return;
  n0 *= kN;
  m0 *= kM;
  const int wn = wave % WN, wm = wave / WN;
  const int my_n = n0 + wn * 16 * TN, my_m = m0 + wm * 16 * TM;
  const int steps = (a.k + kBlock - 1) / kBlock, rest = a.k - (steps - 1) * kBlock;
  const int piece = (lane & 7) ^ (lane >> 3);
  uint32_t woff[kLoadsW], xoff[kLoadsX];
#pragma unroll
  for (int i = 0; i < kLoadsW; ++i)
    woff[i] = (uint32_t)min((wave * kLoadsW + i) * 8 + (lane >> 3), a.n - 1 - n0) * (uint32_t)a.ldw + piece * 16;
#pragma unroll
  for (int i = 0; i < kLoadsX; ++i)
    xoff[i] = (uint32_t)min((wave * kLoadsX + i) * 8 + (lane >> 3), a.m - 1 - m0) * (uint32_t)a.ldx + piece * 16;
  const uint32_t mine = 4u * min(my_m + min(lane, 16 * TM - 1), a.m - 1);
  const float* const ws = a.ws + min(my_n / kBlock, (a.n - 1) / kBlock) * a.ldws;
  float wscale = ws[min(lane, steps - 1)];
  arrived(wscale);
  const uint32_t at0 = lds_address(lds);
  const char* wp = reinterpret_cast<const char*>(a.w) + n0 * a.ldw;
  const char* xp = reinterpret_cast<const char*>(a.x) + m0 * a.ldx;
  const char* sp = reinterpret_cast<const char*>(a.xs);
  int loaded = 0, to = 0;
  // The next block's loads; past the last block the last one's again.
  const auto load = [&]() {
    const uint32_t st = at0 + to * kStage;
    const uint32_t back = loaded == steps - 1 && piece * 16 >= rest ? (uint32_t)(piece * 16 - rest + 16) : 0u;
#pragma unroll
    for (int i = 0; i < kLoadsW; ++i) load16_w<kOnce>(wp, woff[i] - back, st + (wave * kLoadsW + i) * 1024);
#pragma unroll
    for (int i = 0; i < kLoadsX; ++i) load16(xp, xoff[i] - back, st + kN * kBlock + (wave * kLoadsX + i) * 1024);
    load4(sp, mine, st + (kN + kM) * kBlock + wave * 256);
    if (loaded < steps - 1) {
      ++loaded;
      wp += kBlock;
      xp += kBlock;
      sp += a.ldxs * 4;
    }
    to = to == kStages - 1 ? 0 : to + 1;
  };
  const int lo = at * kBlock + ((quarter ^ (at & 7)) * 16), hi = lo ^ 64;
  struct Ops {
    i32x8 w[TN], x[TM];
    float f[TM];
  };
  int from = 0;
  const auto read = [&](Ops& o) {
    const char* const stage = lds + from * kStage;
    const auto operand = [&](int row) {
      const char* const p = stage + row * kBlock;
      return join(*reinterpret_cast<const u32x4*>(p + lo), *reinterpret_cast<const u32x4*>(p + hi));
    };
#pragma unroll
    for (int t = 0; t < TM; ++t) o.x[t] = operand(kN + (wm * TM + t) * 16);
#pragma unroll
    for (int i = 0; i < TN; ++i) o.w[i] = operand((wn * TN + i) * 16);
#pragma unroll
    for (int t = 0; t < TM; ++t) o.f[t] = reinterpret_cast<const float*>(stage + (kN + kM) * kBlock + wave * 256)[16 * t + at];
    from = from == kStages - 1 ? 0 : from + 1;
  };
  f32x4 sum[TN][TM] = {};
  const auto use = [&](Ops& o, int b, bool tail) {
    if (tail) {
#pragma unroll
      for (int i = 0; i < TN; ++i) o.w[i] = cut_off(o.w[i], quarter, rest);
#pragma unroll
      for (int t = 0; t < TM; ++t) o.x[t] = cut_off(o.x[t], quarter, rest);
    }
    if ((b & 63) == 0 && b > 0) {
      wscale = ws[min(b + lane, steps - 1)];
      arrived(wscale);
    }
    const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscale), b & 63));
    f32x4 y[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int t = 0; t < TM; ++t) y[i][t] = mma<kF32Out>(o.w[i], o.x[t]);
    __builtin_amdgcn_sched_barrier(0);
    load();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][t][j] = fmaf(y[i][t][j], o.f[t] * g, sum[i][t][j]);
  };
#pragma unroll
  for (int b = 0; b < kStages; ++b) load();
  Ops one, two;
  wait_loads<(kStages - 1) * kLoads>();
  barrier();
  read(one);
  const auto step = [&](int b, Ops& now, Ops& next) {
    // The next block is there, and everybody has read this one.
    wait_loads<(kStages - 2) * kLoads>();
    wait_lds();
    barrier();
    read(next);
    __builtin_amdgcn_sched_barrier(0);
    use(now, b, b == steps - 1 && rest < kBlock);
  };
  for (int b = 0; b < steps; b += 2) {
    step(b, one, two);
    if (b + 1 < steps) step(b + 1, two, one);
  }
  wait_loads<0>();
  wait_lds();
  barrier();
  store_rows<TN, TM, kF32Out>(a, my_n, my_m, quarter, at, sum, lds + wave * kScratch<TN, TM, kF32Out>);
}

// Many tokens: the matrix cores' rate is what takes time.  A workgroup of WN x WM waves has
// 16 TN WN weight rows and 16 TM WM tokens, a wave 16 TN by 16 TM, of which the weight rows
// lie in one scale block.  A step is a block of k.  Its operands come to LDS without a
// register between, rows of 128 bytes whose 16-byte pieces lie in an order that depends on
// the row, so that the 16 rows of an operand start in different banks.  A step loads the next
// one's weights, and the tokens of the one after that (three places in LDS): a wave reads
// the next step's tokens, which all waves waited for before the barrier at this one's start,
// while it makes this one's last products, and only two reads stand between a barrier and
// the first product after it.  All loads of a step have to be there at its end.  Loads of
// weights two rows of products after those of tokens, not with them: 170 us instead of 179
// at 8192 x 6144 x 4096; a wave that has only four rows loads both at the start (352 and 357).
template <int WN, int WM, int TN, int TM, bool kF32Out>
__global__ __launch_bounds__(64 * WN * WM) void tiles_kernel(MatmulArgs a, int tiles_n, int tiles_m) {
  constexpr int kN = 16 * TN * WN, kM = 16 * TM * WM, kWaves = WN * WM;
  constexpr int kLoadsW = kN / 8 / kWaves, kLoadsX = kM / 8 / kWaves;  // a wave's of a block, 8 rows each
  constexpr int kAhead = 2;                     // weight operands read ahead
  constexpr int kLater = TN > 4 ? 2 : 0;  // the row of products before which weights are loaded
  static_assert(kN % (8 * kWaves) == 0 && kM % (8 * kWaves) == 0 && 16 * TN <= kBlock && TN >= kAhead, "rows");
  constexpr int kW = kN * kBlock, kX = kM * kBlock;  // bytes of a block
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const char* const xlds = lds + 2 * kW;
  const uint32_t at0 = lds_address(lds), xat0 = at0 + 2 * kW;
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, at = lane & 15;
  int n0, m0;
  if (!tile_of(tiles_n, tiles_m, &n0, &m0)) return;
  n0 *= kN;
  m0 *= kM;
  const int wn = wave % WN, wm = wave / WN;
  const int my_n = n0 + wn * 16 * TN, my_m = m0 + wm * 16 * TM;
  const int steps = (a.k + kBlock - 1) / kBlock, rest = a.k - (steps - 1) * kBlock;  // of the last block

  const int piece = (lane & 7) ^ (lane >> 3);
  uint32_t woff[kLoadsW], xoff[kLoadsX];  // rows past the last are read as the last
#pragma unroll
  for (int i = 0; i < kLoadsW; ++i)
    woff[i] = (uint32_t)min((wave * kLoadsW + i) * 8 + (lane >> 3), a.n - 1 - n0) * (uint32_t)a.ldw + piece * 16;
#pragma unroll
  for (int i = 0; i < kLoadsX; ++i)
    xoff[i] = (uint32_t)min((wave * kLoadsX + i) * 8 + (lane >> 3), a.m - 1 - m0) * (uint32_t)a.ldx + piece * 16;
  const char* const wbase = reinterpret_cast<const char*>(a.w) + n0 * a.ldw;
  const char* const xbase = reinterpret_cast<const char*>(a.x) + m0 * a.ldx;
  // In the last block pieces past k are read as its last one, and not used.
  const auto back = [&](int b) { return b == steps - 1 && piece * 16 >= rest ? (uint32_t)(piece * 16 - rest + 16) : 0u; };
  const auto load_w = [&](int b, int half, int i) {
    load16(wbase + b * kBlock, woff[i] - back(b), at0 + half * kW + (wave * kLoadsW + i) * 1024);
  };
  const auto load_x = [&](int b, int third, int i) {
    load16(xbase + b * kBlock, xoff[i] - back(b), xat0 + third * kX + (wave * kLoadsX + i) * 1024);
  };
  const int lo = at * kBlock + ((quarter ^ (at & 7)) * 16), hi = lo ^ 64;
  const auto operand = [&](const char* tile) {
    return join(*reinterpret_cast<const u32x4*>(tile + lo), *reinterpret_cast<const u32x4*>(tile + hi));
  };
  const auto cut = [&](i32x8 v) { return cut_off(v, quarter, rest); };
  // Scales: a lane has one of the wave's tokens, and a weight scale of 64 blocks.
  const uint32_t mine = min(my_m + (lane & (16 * TM - 1)), a.m - 1);
  const float* const ws = a.ws + min(my_n / kBlock, (a.n - 1) / kBlock) * a.ldws;
  float wscale = 0.f;
  const auto token_scale = [&](int b) { return (a.xs + b * a.ldxs)[mine]; };
  const auto factors = [&](float x, int b, float* f) {
    x *= __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscale), b & 63));
    if constexpr (TM == 4) {
      const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(h[i], h[i], false, false);
        f[2 * i] = __uint_as_float(r[0]);
        f[2 * i + 1] = __uint_as_float(r[1]);
      }
    } else if constexpr (TM == 2) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      f[0] = __uint_as_float(r[0]);
      f[1] = __uint_as_float(r[1]);
    } else {
      static_assert(TM == 1 || TM == 2 || TM == 4, "tokens of a wave");
      f[0] = x;
    }
  };

  f32x4 sum[TN][TM] = {}, y[2][TM] = {};
  float f[TM] = {};
#pragma unroll
  for (int i = 0; i < kLoadsW; ++i) load_w(0, 0, i);
#pragma unroll
  for (int i = 0; i < kLoadsX; ++i) load_x(0, 0, i);
#pragma unroll
  for (int i = 0; i < kLoadsX; ++i) load_x(min(1, steps - 1), 1, i);
  float fx = token_scale(0);
  wait_loads<0>();
  barrier();
  const char* const xt = xlds + wm * 16 * TM * kBlock;
  i32x8 xb[TM];
#pragma unroll
  for (int t = 0; t < TM; ++t) xb[t] = operand(xt + t * 16 * kBlock);
  int third = 0;  // b % 3
  const auto step = [&](int b, auto tail) {
    constexpr bool kTail = decltype(tail)::value;
    const char* const wt = lds + (b & 1) * kW + wn * 16 * TN * kBlock;
    const int next = third == 2 ? 0 : third + 1, after = next == 2 ? 0 : next + 1;
    if ((b & 63) == 0) {
      wscale = ws[min(b + lane, steps - 1)];
      arrived(wscale);
    }
    i32x8 wb[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      wb[i] = operand(wt + i * 16 * kBlock);
      if constexpr (kTail) wb[i] = cut(wb[i]);
    }
    if constexpr (kTail) {
#pragma unroll
      for (int t = 0; t < TM; ++t) xb[t] = cut(xb[t]);
    }
    float old[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) old[t] = f[t];
    factors(fx, b, f);
    // Loads past the last block read it again, to places that nobody reads.
    const int b1 = min(b + 1, steps - 1), b2 = min(b + 2, steps - 1);
    if constexpr (!kTail) {
      fx = token_scale(b1);
#pragma unroll
      for (int i = 0; i < kLoadsX; ++i) load_x(b2, after, i);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      if (!kTail && i == kLater) {
#pragma unroll
        for (int l = 0; l < kLoadsW; ++l) load_w(b1, (b + 1) & 1, l);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = 0; t < TM; ++t) {
        y[i & 1][t] = mma<kF32Out>(wb[i % kAhead], xb[t]);
        if (t == TM - 1 && i + kAhead < TN) {
          wb[i % kAhead] = operand(wt + (i + kAhead) * 16 * kBlock);
          if constexpr (kTail) wb[i % kAhead] = cut(wb[i % kAhead]);
        }
        if (!kTail && i == TN - 1) xb[t] = operand(xt + next * kX + t * 16 * kBlock);
        if constexpr (!kF32Out) __builtin_amdgcn_sched_barrier(0);
        // While it is made (32 cycles), four additions of the row before, at first the last
        // step's last row.
        const int r = (i + TN - 1) % TN;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[r][t][j] = fmaf(y[(i + 1) & 1][t][j], i == 0 ? old[t] : f[t], sum[r][t][j]);
        if constexpr (!kF32Out) __builtin_amdgcn_sched_barrier(0);
      }
    }
    third = next;
    // No product stays behind the barrier: with it would the wait for its operands.
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!kTail) {
      wait_loads<0>();
      arrived(fx);
    }
    barrier();
  };
  const int whole = rest == kBlock ? steps : steps - 1;
  for (int b = 0; b < whole; ++b) step(b, std::false_type{});
  if (whole < steps) step(whole, std::true_type{});
  wait_loads<0>();  // nothing comes to LDS any more
  barrier();
#pragma unroll
  for (int t = 0; t < TM; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[TN - 1][t][j] = fmaf(y[(TN - 1) & 1][t][j], f[t], sum[TN - 1][t][j]);
  store_rows<TN, TM, kF32Out>(a, my_n, my_m, quarter, at, sum, lds + wave * kScratch<TN, TM, kF32Out>);
}

template <int WN, int WM, int TN, int TM, typename K>
hipError_t launch(K kernel, int waves, int bytes, std::atomic<uint64_t>& done, const MatmulArgs& a, hipStream_t s) {
  constexpr int kN = 16 * TN * WN, kM = 16 * TM * WM;
  if (bytes > 65536)
    if (const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes, done); e != hipSuccess) return e;
  const int tiles_n = (a.n + kN - 1) / kN, tiles_m = (a.m + kM - 1) / kM;
  kernel<<<(tiles_n * tiles_m + 7) / 8 * 8, 64 * waves, bytes, s>>>(a, tiles_n, tiles_m);
  return hipGetLastError();
}

template <int WN, int WM, int TN, int TM, int kStages, bool kF32Out, bool kOnce = false>
hipError_t launch_small_tiles(const MatmulArgs& a, hipStream_t s) {
  if constexpr (!kOnce)
    if (a.m <= 16 * TM * WM) return launch_small_tiles<WN, WM, TN, TM, kStages, kF32Out, true>(a, s);
  constexpr int kBytes = kStages * (16 * (TN * WN + TM * WM) * kBlock + WN * WM * 256);
  static_assert(kBytes >= WN * WM * kScratch<TN, TM, kF32Out>, "results in LDS");
  static std::atomic<uint64_t> done{0};
  return launch<WN, WM, TN, TM>(small_tiles_kernel<WN, WM, TN, TM, kStages, kF32Out, kOnce>, WN * WM, kBytes, done, a, s);
}

template <int WN, int WM, int TN, int TM, bool kF32Out>
hipError_t launch_tiles(const MatmulArgs& a, hipStream_t s) {
  constexpr int kOps = 16 * (2 * TN * WN + 3 * TM * WM) * kBlock, kOut = WN * WM * kScratch<TN, TM, kF32Out>;
  constexpr int kBytes = kOps > kOut ? kOps : kOut;
  static std::atomic<uint64_t> done{0};
  return launch<WN, WM, TN, TM>(tiles_kernel<WN, WM, TN, TM, kF32Out>, WN * WM, kBytes, done, a, s);
}

template <int TN, bool kF32Out>
hipError_t launch_few(const MatmulArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  return launch<1, 1, TN, 1>(few_tokens_kernel<TN, kF32Out>, 8, 0, done, a, s);
}

template <int TN, int TM, int kAhead, int kWaves, bool kF32Out, bool kOnce = false>
hipError_t launch_stream(const MatmulArgs& a, hipStream_t s) {
  if constexpr (!kOnce)
    if (a.m <= 16 * TM) return launch_stream<TN, TM, kAhead, kWaves, kF32Out, true>(a, s);
  constexpr int kBytes = kWaves * kAhead * (16 * (TN + TM) * kBlock + 256);
  static_assert(kBytes >= kWaves * TN * TM * 1024, "sums in LDS");
  static std::atomic<uint64_t> done{0};
  return launch<1, 1, TN, TM>(stream_kernel<TN, TM, kAhead, kWaves, kF32Out, kOnce>, kWaves, kBytes, done, a, s);
}

// What a form takes, in us: base + load * wave + a step's greater of alone and load *
// shared, a step, with load the tiles of the busiest compute unit, and not less than 3 +
// its weights and results at `rate` MB/us.  Fitted to 326 sizes for each type of result (1
// to 4096 tokens, 512 to 32000 weight rows, k from 512 to 6144; weights from memory, as a
// model's layers find them), foremost to which form is fastest.  The one chosen takes 0.3 %
// more than the best on average there, 16 % at most (sizes left out of the fit: 0.5 and
// 19 %).  fp32 results have no 256 x 256, whose operands in fp16 would not fit beside the
// sums, no second 128 x 128 and no 64 x 128, which nothing is faster by.
struct Form {
  int n, m;  // of a tile
  float base, wave, alone, shared, rate;
};
constexpr int kForms = 12;
constexpr Form kBf16Forms[kForms] = {
    {256, 256, 1.09f, 5.28f, 0.229f, 1.4f, 3.91f},
    {128, 128, 1.79f, 1.71f, 1.06f, 0.532f, 3.73f},
    {128, 128, 1.24f, 3.73f, 0.23f, 0.642f, 6.01f},
    {64, 64, 1.51f, 1.22f, 0.353f, 0.278f, 5.76f},
    {32, 32, 1.57f, 1.21f, 0.203f, 0.128f, 4.77f},
    {64, 16, 3.04f, 0.0837f, 0.192f, 0.321f, 4.86f},
    {64, 32, 1.17f, 3.15f, 0.137f, 0.197f, 4.36f},
    {32, 32, 1.22f, 2.68f, 0.0804f, 0.126f, 4.99f},
    {32, 16, 1.46f, 1.35f, 0.117f, 0.13f, 6.4f},
    {16, 16, 2.14f, 1.48f, 0.0638f, 0.0543f, 4.93f},
    {64, 96, 1.29f, 1.31f, 0.529f, 0.388f, 4.99f},
    {64, 128, 1.08f, 2.8f, 0.0914f, 0.416f, 4.51f}};
constexpr Form kF32Forms[kForms] = {
    {256, 256, 1e30f, 0.f, 0.f, 0.f, 1.f},
    {128, 128, 5.02f, 0.973f, 0.332f, 0.831f, 3.64f},
    {128, 128, 1e30f, 0.f, 0.f, 0.f, 1.f},
    {64, 64, 1.92f, 1.14f, 0.576f, 0.374f, 4.74f},
    {32, 32, 1.29f, 1.03f, 0.35f, 0.212f, 5.04f},
    {64, 16, 2.57f, 0.563f, 0.31f, 0.294f, 5.83f},
    {64, 32, 1.4f, 4.04f, 0.176f, 0.212f, 5.63f},
    {32, 32, 1.f, 2.53f, 0.0637f, 0.165f, 4.77f},
    {32, 16, 1.41f, 1.46f, 0.0977f, 0.116f, 6.4f},
    {16, 16, 1.99f, 1.64f, 0.0528f, 0.0499f, 4.84f},
    {64, 96, 1.42f, 1.68f, 0.69f, 0.433f, 3.98f},
    {64, 128, 1e30f, 0.f, 0.f, 0.f, 1.f}};

int choose(const MatmulArgs& a, int m, float* us) {
  const Form* const forms = a.f32 ? kF32Forms : kBf16Forms;
  const int steps = (a.k + kBlock - 1) / kBlock;
  const float mb = ((float)a.n * a.k + (float)m * a.n * (a.f32 ? 4 : 2)) * 1e-6f;
  int best = 1;
  *us = INFINITY;
  for (int i = 0; i < kForms; ++i) {
    const Form& f = forms[i];
    const int64_t tiles = (int64_t)((a.n + f.n - 1) / f.n) * ((m + f.m - 1) / f.m);
    if (i > 1 && tiles > 1 << 22) continue;  // a launch has less than 2^32 threads
    const float load = (float)((tiles + 255) / 256);
    const float t = fmaxf(f.base + f.wave * load + steps * fmaxf(f.alone, load * f.shared), 3.f + mb / f.rate);
    if (t < *us) {
      *us = t;
      best = i;
    }
  }
  return best;
}

template <bool kF32Out>
hipError_t launch_form(int form, const MatmulArgs& a, hipStream_t s) {
  switch (form) {
    case 0:
      if constexpr (!kF32Out) return launch_tiles<2, 4, 8, 4, kF32Out>(a, s);
      [[fallthrough]];
    case 2:
      if constexpr (!kF32Out) return launch_small_tiles<2, 4, 4, 2, 3, kF32Out>(a, s);
      [[fallthrough]];
    case 11:
      if constexpr (!kF32Out) return launch_small_tiles<2, 4, 2, 2, 4, kF32Out>(a, s);
      [[fallthrough]];
    case 1: return launch_tiles<2, 2, 4, 4, kF32Out>(a, s);
    case 3: return launch_small_tiles<2, 2, 2, 2, 4, kF32Out>(a, s);
    case 4: return launch_small_tiles<2, 2, 1, 1, 6, kF32Out>(a, s);
    case 5: return launch_few<4, kF32Out>(a, s);
    case 6: return launch_stream<4, 2, 2, 4, kF32Out>(a, s);
    case 7: return launch_stream<2, 2, 4, 4, kF32Out>(a, s);
    case 8: return launch_stream<2, 1, 2, 4, kF32Out>(a, s);
    case 10: return launch_small_tiles<2, 2, 2, 3, 3, kF32Out>(a, s);
    default: return launch_stream<1, 1, 2, 8, kF32Out>(a, s);
  }
}

hipError_t launch_part(int form, const MatmulArgs& a, hipStream_t s) {
  return a.f32 ? launch_form<true>(form, a, s) : launch_form<false>(form, a, s);
}

}  // namespace

hipError_t launch_scaled_matmul(const MatmulArgs& a, hipStream_t s) {
  float whole, most, few;
  const int form = choose(a, a.m, &whole);
  // A few tokens past whole tiles would take another round of those: a launch of their own,
  // which hides all but about 1 us of its start behind the first.
  const int tail = a.m % 256;
  if (tail != 0 && tail < a.m) {
    const int first = choose(a, a.m - tail, &most), second = choose(a, tail, &few);
    if (most + few - 2.f < whole) {
      MatmulArgs p = a;
      p.m = a.m - tail;
      if (const hipError_t e = launch_part(first, p, s); e != hipSuccess) return e;
      p.m = tail;
      p.x += (a.m - tail) * a.ldx;
      p.xs += a.m - tail;
      p.out += (a.m - tail) * a.ldo * (a.f32 ? 4 : 2);
      return launch_part(second, p, s);
    }
  }
  return launch_part(form, a, s);
}

}  // namespace s2moe
