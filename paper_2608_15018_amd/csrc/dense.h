// Internal launch interface of the norm, the quantization and the 8-bit product.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace s2moe {

constexpr int kBlock = 128;             // elements of a row that share a scale
constexpr float kLargest = 448.f;       // of e4m3
constexpr float kLeast = 0x1p-100f;     // least magnitude that a scale stands for
constexpr int kMaxHidden = 16384;       // of a norm: a row stays in a workgroup's registers

enum : int { kF32 = 0, kBf16 = 1, kE4m3 = 3, kNone = -1 };

struct NormArgs {
  int n, H;
  const char* x;
  char* residual;
  const char* weight;
  char* out;
  float* scales;
  int64_t ldx, ldr, ldo, lds;  // elements
  int x_type, r_type, w_type, out_type;
  float eps;
};
hipError_t launch_add_norm(const NormArgs& a, hipStream_t s);

struct QuantizeArgs {
  int n, cols;
  const char* x;
  char* codes;
  float* scales;
  int64_t ldx, ldc, lds;  // elements
  int x_type;
};
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s);
// Blocks of 128 rows too; scales [ceil(n / 128)][lds].
hipError_t launch_quantize_weight(const QuantizeArgs& a, hipStream_t s);

struct MatmulArgs {
  int m, n, k;
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  char* out;
  int64_t ldx, ldxs, ldw, ldws, ldo;  // elements
  bool f32;                           // out
};
hipError_t launch_scaled_matmul(const MatmulArgs& a, hipStream_t s);

}  // namespace s2moe
