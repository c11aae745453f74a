// Device helpers shared by the attention kernels (gfx950, wave64).
#pragma once

#include "common.h"

namespace s2moe {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// p[i] by a scalar load where i is the same in all lanes; nothing writes p while
// the kernel runs.
__device__ __forceinline__ int constant(const int32_t* p, int64_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p))[i];
}

// A running maximum may lag behind by this much (base-2 logarithm) before the
// accumulators are rescaled: weights stay below 2^8, far inside fp32 and of
// the same relative precision in bf16.
constexpr float kLag = 8.f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  return fmaxf(fmaxf(a, b), c);
}

// The other half-wave's value combined with this one's: lanes l and l ^ 32.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Over the four 16-lane groups.
__device__ __forceinline__ float max_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ bf16x8 pack8(const float* x) {
  bf16x8 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 v = {x[2 * i], x[2 * i + 1]};
    const bf16x2 b = __builtin_convertvector(v, bf16x2);
    out[2 * i] = b[0];
    out[2 * i + 1] = b[1];
  }
  return out;
}

// 16 bytes per lane from base + off (off per lane) to 1 KB of LDS at `lds`,
// lane after lane, without a register between.  In asm, because the compiler
// would wait for every such load before the next read of LDS; whoever reads
// the data waits for it by count and passes a barrier first.  (The compiler warns that
// m0 is reserved; named, it is not expected to hold a value across the statement.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, const char* lds) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(at), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N are in flight
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Until this wave's reads of LDS are done: before a barrier after which other
// waves load over what was read.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

__device__ __forceinline__ bf16x2 pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_convertvector(v, bf16x2);
}

// Nonzero where x holds an infinity or NaN: the top bit of each such element (an
// exponent of ones, and only that, carries into it).
__device__ __forceinline__ uint32_t nonfinite_bits(uint32_t two) {
  return ((two & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
__device__ __forceinline__ uint32_t any_nonfinite(bf16x8 x) {
  const u32x4 u = __builtin_bit_cast(u32x4, x);
  return nonfinite_bits(u[0]) | nonfinite_bits(u[1]) | nonfinite_bits(u[2]) | nonfinite_bits(u[3]);
}
__device__ __forceinline__ uint32_t any_nonfinite(f32x4 x) {
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad |= ((__float_as_uint(x[i]) & 0x7F800000u) + 0x00800000u) & 0x80000000u;
  return bad;
}
// x with those elements zero.
__device__ __forceinline__ bf16x8 finite_only(bf16x8 x) {
  u32x4 u = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = nonfinite_bits(u[i]) >> 15;
    u[i] &= ~((t << 16) - t);  // a bit becomes its half's sixteen
  }
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ f32x4 finite_only(f32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if ((__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u) x[i] = 0.f;
  return x;
}
// What a product with such elements gives, where some weights are zero because a row
// does not see the key: each element as a number (infinity 1, minus infinity 2^8, NaN
// 2^16, finite 0), times 1 for a key that the row sees, 2^16 if its weight has
// underflowed to zero, 0 for one that it does not see.  Up to 32 keys add up, in any
// order, to a number that tells what there was.
constexpr float kNan = 65536.f;
__device__ __forceinline__ bf16x8 special_numbers(bf16x8 x) {
  u32x4 u = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = nonfinite_bits(u[i]) >> 15;  // a bit for each half
    const uint32_t nan = t & (((u[i] & 0x007F007Fu) + 0x007F007Fu) >> 7), minus = t & (u[i] >> 15) & ~nan;
    u[i] = t * 0x3F80u + minus * (0x4380u - 0x3F80u) + nan * (0x4780u - 0x3F80u);
  }
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ f32x4 special_numbers(f32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = x[i] != x[i] ? kNan : x[i] == INFINITY ? 1.f : x[i] == -INFINITY ? 256.f : 0.f;
  return x;
}
// What the weights become there: bit e of `seen` is element e's key.
__device__ __forceinline__ bf16x8 sight(uint32_t seen, bf16x8 weights) {
  u32x4 u = __builtin_bit_cast(u32x4, weights);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t weighs = (((u[i] & 0x7FFF7FFFu) + 0x7FFF7FFFu) >> 15) & 0x00010001u;
    const uint32_t two = (seen >> (2 * i) & 1) | (seen >> (2 * i + 1) & 1) << 16;
    u[i] = (0x47804780u - weighs * (0x4780u - 0x3F80u)) & (two * 0xFFFFu);
  }
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ f32x4 sight(uint32_t seen, f32x4 weights) {
#pragma unroll
  for (int i = 0; i < 4; ++i) weights[i] = !(seen >> i & 1) ? 0.f : weights[i] == 0.f ? kNan : 1.f;
  return weights;
}
__device__ __forceinline__ float special_sum(float number) {
  const int n = number >= kNan ? 0x101 : (int)number;
  const float plus = (n & 255) != 0 ? INFINITY : 0.f, minus = n >> 8 != 0 ? -INFINITY : 0.f;
  return plus + minus;  // NaN where both are there
}

}  // namespace s2moe
