// Rows added to the residual stream and normalised, and rows and weights in 8 bits.
//
//   h = x + r,  r <- h,  y = h * w / sqrt(mean(h^2) + eps)
//
// in fp32 from the loads to one rounding of each output.  In 8 bits a block of 128
// elements has one scale s = max(|y|, 2^-100) / 448, so that its largest element becomes
// e4m3's largest, and the codes are y / s.  A row is read once: it stays in registers
// between the sum of squares and the outputs, a workgroup a row (a wave, up to 512
// columns), eight elements a lane at a time, so that sixteen lanes have a block.
//
// Bound: memory.  8193 rows of 4096, bf16 in, bf16 residual, 8 bits out: 42 us, 5.6 TB/s
// (a large copy: 5.2; with x read through the caches 47, the residual past them too 43,
// stores past them 45); 12289 rows of 4096 from bf16 to 8 bits 30 us, 5.1 TB/s (31 through
// the caches); 251 rows of 2880 with an fp32 residual 4.2 us, a single row 2.3.
#include <type_traits>

#include "attn_common.h"
#include "dense.h"

namespace s2moe {
namespace {

template <int N>
__device__ __forceinline__ float ror(float x) {  // from N lanes on, within 16 lanes
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + N, 0xF, 0xF, true));
}
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, ror<8>(x));
  x = fmaxf(x, ror<4>(x));
  x = fmaxf(x, ror<2>(x));
  return fmaxf(x, ror<1>(x));
}
__device__ __forceinline__ float sum16(float x) {
  x += ror<8>(x);
  x += ror<4>(x);
  x += ror<2>(x);
  return x + ror<1>(x);
}

// Eight neighbouring elements of a row; past the caches where nothing reads or writes them
// again (not a residual).
template <int T>
struct Raw {
  u32x4 v[T == kF32 ? 2 : 1];
};
template <int T, bool kOnce = true>
__device__ __forceinline__ Raw<T> load8(const char* row, int col) {
  Raw<T> r;
  const u32x4* p = reinterpret_cast<const u32x4*>(row + (int64_t)col * (T == kF32 ? 4 : 2));
#pragma unroll
  for (int i = 0; i < (T == kF32 ? 2 : 1); ++i) r.v[i] = kOnce ? __builtin_nontemporal_load(p + i) : p[i];
  return r;
}
template <int T>
__device__ __forceinline__ void floats(const Raw<T>& r, float* f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (T == kF32)
      f[i] = __uint_as_float(r.v[i / 4][i % 4]);
    else
      f[i] = __uint_as_float(i & 1 ? r.v[0][i / 2] & 0xFFFF0000u : r.v[0][i / 2] << 16);
  }
}
template <int T>
__device__ __forceinline__ void store8(char* row, int col, const float* f) {
  if constexpr (T == kF32) {
    f32x4* p = reinterpret_cast<f32x4*>(row + (int64_t)col * 4);
    p[0] = f32x4{f[0], f[1], f[2], f[3]};
    p[1] = f32x4{f[4], f[5], f[6], f[7]};
  } else {
    *reinterpret_cast<bf16x8*>(row + (int64_t)col * 2) = pack8(f);
  }
}

// Eight elements z, which are at most 448 and a rounding of fp32: e4m3 rounds that to 448.
__device__ __forceinline__ uint2 codes8(const float* z) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[4], z[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[6], z[7], hi, true);
  return uint2{(uint32_t)lo, (uint32_t)hi};
}

// 448 y / most.  Of elements of few bits (bf16) one quotient in 200 is half way between two codes,
// and 448 / most rounded to fp32 would take up to a sixth of those to the other code than
// the even one.  So it has two parts: 16 bits, whose product with such an element is exact,
// and the rest, 22 more; the sum is rounded once.  As 7/8 over most / 512, whose reciprocal
// is never below fp32's normal range.
__device__ __forceinline__ void divide8(float* y, float most) {
  const float d = most * 0x1p-9f, r = __builtin_amdgcn_rcpf(d);
  const float top = __uint_as_float(__float_as_uint(0.875f * r) & 0xFFFFFF00u), rest = fmaf(-top, d, 0.875f) * r;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fmaf(y[i], rest, y[i] * top);
}

__device__ __forceinline__ float most8(const float* y) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(y[i]));
  return top;
}

// Codes and scale of a block, sixteen lanes' eight elements each, which `most` is the largest
// of.  `live` lanes have elements, the others zeros.
__device__ __forceinline__ void store_block(char* codes, float* scales, int64_t lds, int row, int col, bool live,
                                            const float* z, float most) {
  if (!live) return;
  *reinterpret_cast<uint2*>(codes + col) = codes8(z);
  if ((threadIdx.x & 15) == 0) scales[(col / kBlock) * lds + row] = most / kLargest;
}

// kLanes lanes a row (64, or the whole workgroup), kChunks times eight elements each.
template <int X, int R, int O, int kLanes, int kChunks>
__global__ __launch_bounds__(256) void add_norm_kernel(NormArgs a) {
  __shared__ float part[4];
  const int lane = threadIdx.x % kLanes;
  const int row0 = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const int row = min(row0, a.n - 1);
  const bool mine = row0 < a.n;
  const char* x = a.x + row * a.ldx * (X == kF32 ? 4 : 2);
  char* r = R == kNone ? nullptr : a.residual + row * a.ldr * (R == kF32 ? 4 : 2);
  Raw<X> xs[kChunks];
  Raw<R == kNone ? kBf16 : R> rs[kChunks];
  u32x4 ws[kChunks][2];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int col = (c * kLanes + lane) * 8;
    if (col < a.H) {
      xs[c] = load8<X>(x, col);
      if constexpr (R != kNone) rs[c] = load8<R, false>(r, col);
      if (a.w_type == kF32) {
        ws[c][0] = reinterpret_cast<const u32x4*>(a.weight)[col / 4];
        ws[c][1] = reinterpret_cast<const u32x4*>(a.weight)[col / 4 + 1];
      } else {
        ws[c][0] = reinterpret_cast<const u32x4*>(a.weight)[col / 8];
      }
    }
  }
  float h[kChunks][8], sum = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int col = (c * kLanes + lane) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[c][i] = 0.f;
    if (col < a.H) {
      floats<X>(xs[c], h[c]);
      if constexpr (R != kNone) {
        float old[8];
        floats<R>(rs[c], old);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] += old[i];
        if (mine) store8<R>(r, col, h[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(h[c][i], h[c][i], sum);
    }
  }
  sum = sum_groups(sum16(sum));
  if constexpr (kLanes > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const float norm = 1.f / sqrtf(sum / (float)a.H + a.eps);
  if (!mine) return;
  // The norm's power of two and what is left of it, between 1 and 2.
  const float power = __uint_as_float(__float_as_uint(norm) & 0x7F800000u), left = norm / power;
  char* out = a.out + row * a.ldo * (O == kF32 ? 4 : O == kBf16 ? 2 : 1);
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int col = (c * kLanes + lane) * 8;
    const bool live = col < a.H;
    float y[8] = {};
    if (live) {
      float w[8];
      if (a.w_type == kF32)
        floats<kF32>(Raw<kF32>{{ws[c][0], ws[c][1]}}, w);
      else
        floats<kBf16>(Raw<kBf16>{{ws[c][0]}}, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[c][i] * (O == kE4m3 ? power : norm) * w[i];
    }
    if constexpr (O == kE4m3) {
      // The norm divides a block's elements and its largest alike: the codes are 448 h w over
      // the largest |h w|, and the norm's own rounding does not reach them.  Its power of two
      // does, exactly, so that h w is as far from the ends of fp32 as y is.  Of blocks below
      // the least magnitude it is 448 y over that.
      const float top = max16(most8(y)), most = fmaxf(top * left, kLeast);
      divide8(y, most > kLeast ? top : fminf(kLeast / left, 3e38f));
      store_block(out, a.scales, a.lds, row, col, live, y, most);
    } else {
      if (live) store8<O>(out, col, y);
    }
  }
}

// A wave takes 512 columns of a row.
template <int X>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a) {
  const int lane = threadIdx.x & 63, parts = (a.cols + 511) / 512;
  const int64_t all = (int64_t)a.n * parts;
  for (int64_t at = (int64_t)blockIdx.x * 4 + wave_id(); at < all; at += (int64_t)gridDim.x * 4) {
    const int row = (int)(at / parts), col = (int)(at % parts) * 512 + lane * 8;
    const bool live = col < a.cols;
    float y[8] = {};
    if (live) floats<X>(load8<X>(a.x + row * a.ldx * (X == kF32 ? 4 : 2), col), y);
    const float most = fmaxf(max16(most8(y)), kLeast);
    divide8(y, most);
    store_block(a.codes + row * a.ldc, a.scales, a.lds, row, col, live, y, most);
  }
}

// A workgroup takes a block: sixteen lanes a row, sixteen rows at a time.
template <int X>
__global__ __launch_bounds__(256) void quantize_weight_kernel(QuantizeArgs a) {
  __shared__ float part[4];
  const int col = blockIdx.x * kBlock + (threadIdx.x & 15) * 8;
  const int row0 = blockIdx.y * kBlock + (threadIdx.x >> 4);
  float y[8][8] = {}, top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 16 * i;
    if (row < a.n && col < a.cols) floats<X>(load8<X>(a.x + row * a.ldx * (X == kF32 ? 4 : 2), col), y[i]);
    top = fmaxf(top, most8(y[i]));
  }
  top = max_groups(max16(top));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const float most = fmaxf(top, kLeast);
  if (threadIdx.x == 0) a.scales[blockIdx.y * a.lds + blockIdx.x] = most / kLargest;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 16 * i;
    divide8(y[i], most);
    if (row < a.n && col < a.cols) *reinterpret_cast<uint2*>(a.codes + row * a.ldc + col) = codes8(y[i]);
  }
}

template <int T>
using Type = std::integral_constant<int, T>;

template <typename F>
void by_float(int type, F f) {
  if (type == kF32) f(Type<kF32>{});
  else f(Type<kBf16>{});
}

template <int X, int R, int O>
void launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.H <= 512) add_norm_kernel<X, R, O, 64, 1><<<(a.n + 3) / 4, 256, 0, s>>>(a);
  else if (a.H <= 2048) add_norm_kernel<X, R, O, 256, 1><<<a.n, 256, 0, s>>>(a);
  else if (a.H <= 4096) add_norm_kernel<X, R, O, 256, 2><<<a.n, 256, 0, s>>>(a);
  else if (a.H <= 8192) add_norm_kernel<X, R, O, 256, 4><<<a.n, 256, 0, s>>>(a);
  else add_norm_kernel<X, R, O, 256, 8><<<a.n, 256, 0, s>>>(a);
}

}  // namespace

hipError_t launch_add_norm(const NormArgs& a, hipStream_t s) {
  by_float(a.x_type, [&](auto x) {
    const auto with = [&](auto r) {
      constexpr int X = decltype(x)::value, R = decltype(r)::value;
      if (a.out_type == kE4m3) launch_norm<X, R, kE4m3>(a, s);
      else if (a.out_type == kF32) launch_norm<X, R, kF32>(a, s);
      else launch_norm<X, R, kBf16>(a, s);
    };
    if (a.r_type == kNone) with(Type<kNone>{});
    else by_float(a.r_type, with);
  });
  return hipGetLastError();
}

hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  const int64_t groups = ((int64_t)a.n * ((a.cols + 511) / 512) + 3) / 4;
  const unsigned grid = groups < 1 << 20 ? (unsigned)groups : 1 << 20;
  by_float(a.x_type, [&](auto x) { quantize_kernel<decltype(x)::value><<<grid, 256, 0, s>>>(a); });
  return hipGetLastError();
}

hipError_t launch_quantize_weight(const QuantizeArgs& a, hipStream_t s) {
  const dim3 grid((a.cols + kBlock - 1) / kBlock, (a.n + kBlock - 1) / kBlock);
  by_float(a.x_type, [&](auto x) { quantize_weight_kernel<decltype(x)::value><<<grid, 256, 0, s>>>(a); });
  return hipGetLastError();
}

}  // namespace s2moe
