// C-ABI entry points of the norm, the quantization and the 8-bit product: argument
// checks on the host, then kernel launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dense.h"
#include "rows.h"
#include "s2moe.h"
#include "status.h"

static_assert((int)s2moe::kF32 == (int)S2MOE_F32 && (int)s2moe::kBf16 == (int)S2MOE_BF16 &&
                  (int)s2moe::kE4m3 == (int)S2MOE_E4M3,
              "dtypes");
static_assert(s2moe::kBlock == S2MOE_SCALE_BLOCK, "block of a scale");

namespace {

using s2moe::aligned;
using s2moe::aligned16;
using s2moe::bytes_meet;
using s2moe::fail;
using s2moe::hip_status;
using s2moe::ok;
using s2moe::rows_meet;

constexpr int kMaxRows = 1 << 22;
constexpr int kMaxCols = 1 << 18;

int elt(int dtype) { return dtype == S2MOE_F32 ? 4 : dtype == S2MOE_BF16 ? 2 : 1; }

bool is_float(int dtype) { return dtype == S2MOE_F32 || dtype == S2MOE_BF16; }

s2moe_status check_count(const char* fn, const char* name, int32_t n, int32_t least, int32_t most) {
  if (n < least) return fail(S2MOE_EINVAL, "%s: %s = %d < %d", fn, name, n, least);
  if (n > most) return fail(S2MOE_EUNSUPPORTED, "%s: %s = %d exceeds %d", fn, name, n, most);
  return S2MOE_OK;
}

// Columns, which the kernels take 16 at a time.
s2moe_status check_cols(const char* fn, const char* name, int32_t n, int32_t most) {
  const s2moe_status st = check_count(fn, name, n, 1, most);
  if (st == S2MOE_OK && n % 16 != 0)
    return fail(S2MOE_EINVAL, "%s: %s = %d is not a multiple of 16", fn, name, n);
  return st;
}

s2moe_status check_stride(const char* fn, const char* name, int64_t ld, int64_t cols, int size) {
  if (ld < cols)
    return fail(S2MOE_EINVAL, "%s: %s = %lld < %lld", fn, name, (long long)ld, (long long)cols);
  if (ld > (int64_t)1 << 22)
    return fail(S2MOE_EUNSUPPORTED, "%s: %s = %lld exceeds 2^22 elements", fn, name, (long long)ld);
  if (size > 0 && ld * size % 16 != 0)
    return fail(S2MOE_EINVAL, "%s: %s = %lld elements is not a multiple of 16 bytes", fn, name,
                (long long)ld);
  return S2MOE_OK;
}

// Bytes that `rows` rows of `width` elements every `ld` stretch over.
int64_t extent(int64_t rows, int64_t ld, int64_t width, int size) {
  return ((rows - 1) * ld + width) * size;
}

int64_t blocks(int64_t n) { return (n + S2MOE_SCALE_BLOCK - 1) / S2MOE_SCALE_BLOCK; }

}  // namespace

extern "C" {

s2moe_status s2moe_add_norm(int32_t n, int32_t hidden, const void* x, int64_t ldx, int32_t x_dtype,
                            void* residual, int64_t ldr, int32_t r_dtype, const void* weight,
                            int32_t w_dtype, float eps, void* out, int64_t ldo, int32_t out_dtype,
                            float* scales, int64_t lds, void* stream) {
  const char* fn = "s2moe_add_norm";
  s2moe_status st = check_count(fn, "n", n, 0, kMaxRows);
  if (st == S2MOE_OK) st = check_cols(fn, "hidden", hidden, s2moe::kMaxHidden);
  if (st != S2MOE_OK) return st;
  if (!is_float(x_dtype))
    return fail(S2MOE_EINVAL, "%s: x_dtype = %d must be F32 or BF16", fn, x_dtype);
  if (!is_float(w_dtype))
    return fail(S2MOE_EINVAL, "%s: w_dtype = %d must be F32 or BF16", fn, w_dtype);
  if (residual != nullptr && !is_float(r_dtype))
    return fail(S2MOE_EINVAL, "%s: r_dtype = %d must be F32 or BF16", fn, r_dtype);
  if (!is_float(out_dtype) && out_dtype != S2MOE_E4M3)
    return fail(S2MOE_EINVAL, "%s: out_dtype = %d must be F32, BF16 or E4M3", fn, out_dtype);
  if (!std::isfinite(eps) || !(eps > 0.f))
    return fail(S2MOE_EINVAL, "%s: eps = %g must be finite and > 0", fn, (double)eps);
  if (n == 0) return ok();
  const bool codes = out_dtype == S2MOE_E4M3;
  S2MOE_REQUIRE_PTR(x);
  S2MOE_REQUIRE_PTR(weight);
  S2MOE_REQUIRE_PTR(out);
  if ((st = check_stride(fn, "ldx", ldx, hidden, elt(x_dtype))) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldo", ldo, hidden, elt(out_dtype))) != S2MOE_OK) return st;
  const int64_t wx = (int64_t)hidden * elt(x_dtype), wo = (int64_t)hidden * elt(out_dtype);
  const int64_t sx = ldx * elt(x_dtype), so = ldo * elt(out_dtype);
  const int64_t ww = (int64_t)hidden * elt(w_dtype), eo = extent(n, ldo, hidden, elt(out_dtype));
  if (rows_meet(x, sx, wx, out, so, wo, n)) return fail(S2MOE_EINVAL, "%s: out overlaps x", fn);
  if (bytes_meet(weight, ww, out, eo))
    return fail(S2MOE_EINVAL, "%s: out overlaps weight", fn);
  const int64_t es = codes ? extent(blocks(hidden), lds, n, 4) : 0;
  if (codes) {
    S2MOE_REQUIRE_INTS(scales);
    if ((st = check_stride(fn, "lds", lds, n, 0)) != S2MOE_OK) return st;
    if (bytes_meet(scales, es, x, extent(n, ldx, hidden, elt(x_dtype))) ||
        bytes_meet(scales, es, out, eo) || bytes_meet(scales, es, weight, ww))
      return fail(S2MOE_EINVAL, "%s: scales overlap x, weight or out", fn);
  }
  if (residual != nullptr) {
    if (!aligned16(residual))
      return fail(S2MOE_EINVAL, "%s: residual is not 16-byte aligned", fn);
    if ((st = check_stride(fn, "ldr", ldr, hidden, elt(r_dtype))) != S2MOE_OK) return st;
    const int64_t wr = (int64_t)hidden * elt(r_dtype), sr = ldr * elt(r_dtype);
    const int64_t er = extent(n, ldr, hidden, elt(r_dtype));
    if (rows_meet(x, sx, wx, residual, sr, wr, n) || rows_meet(out, so, wo, residual, sr, wr, n) ||
        bytes_meet(weight, ww, residual, er) || (codes && bytes_meet(scales, es, residual, er)))
      return fail(S2MOE_EINVAL, "%s: residual overlaps x, weight, out or scales", fn);
  }
  s2moe::NormArgs a;
  a.n = n;
  a.H = hidden;
  a.x = static_cast<const char*>(x);
  a.residual = static_cast<char*>(residual);
  a.weight = static_cast<const char*>(weight);
  a.out = static_cast<char*>(out);
  a.scales = scales;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldo = ldo;
  a.lds = lds;
  a.x_type = x_dtype;
  a.r_type = residual == nullptr ? (int)s2moe::kNone : r_dtype;
  a.w_type = w_dtype;
  a.out_type = out_dtype;
  a.eps = eps;
  return hip_status(fn, s2moe::launch_add_norm(a, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_quantize(int32_t n, int32_t cols, const void* x, int64_t ldx, int32_t x_dtype,
                            void* codes, int64_t ldc, float* scales, int64_t lds, void* stream) {
  const char* fn = "s2moe_quantize";
  s2moe_status st = check_count(fn, "n", n, 0, kMaxRows);
  if (st == S2MOE_OK) st = check_cols(fn, "cols", cols, kMaxCols);
  if (st != S2MOE_OK) return st;
  if (!is_float(x_dtype))
    return fail(S2MOE_EINVAL, "%s: x_dtype = %d must be F32 or BF16", fn, x_dtype);
  if (n == 0) return ok();
  S2MOE_REQUIRE_PTR(x);
  S2MOE_REQUIRE_PTR(codes);
  S2MOE_REQUIRE_INTS(scales);
  const int ex = elt(x_dtype);
  if ((st = check_stride(fn, "ldx", ldx, cols, ex)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldc", ldc, cols, 1)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "lds", lds, n, 0)) != S2MOE_OK) return st;
  const int64_t es = extent(blocks(cols), lds, n, 4);
  if (rows_meet(x, ldx * ex, (int64_t)cols * ex, codes, ldc, cols, n) ||
      bytes_meet(scales, es, x, extent(n, ldx, cols, ex)) ||
      bytes_meet(scales, es, codes, extent(n, ldc, cols, 1)))
    return fail(S2MOE_EINVAL, "%s: x, codes and scales overlap", fn);
  s2moe::QuantizeArgs a;
  a.n = n;
  a.cols = cols;
  a.x = static_cast<const char*>(x);
  a.codes = static_cast<char*>(codes);
  a.scales = scales;
  a.ldx = ldx;
  a.ldc = ldc;
  a.lds = lds;
  a.x_type = x_dtype;
  return hip_status(fn, s2moe::launch_quantize(a, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_quantize_weight(int32_t rows, int32_t cols, const void* w, int64_t ldw,
                                   int32_t w_dtype, void* codes, int64_t ldc, float* scales,
                                   int64_t lds, void* stream) {
  const char* fn = "s2moe_quantize_weight";
  s2moe_status st = check_count(fn, "rows", rows, 1, kMaxRows);
  if (st == S2MOE_OK) st = check_cols(fn, "cols", cols, kMaxCols);
  if (st != S2MOE_OK) return st;
  if (!is_float(w_dtype))
    return fail(S2MOE_EINVAL, "%s: w_dtype = %d must be F32 or BF16", fn, w_dtype);
  S2MOE_REQUIRE_PTR(w);
  S2MOE_REQUIRE_PTR(codes);
  S2MOE_REQUIRE_INTS(scales);
  const int ew = elt(w_dtype);
  if ((st = check_stride(fn, "ldw", ldw, cols, ew)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldc", ldc, cols, 1)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "lds", lds, blocks(cols), 0)) != S2MOE_OK) return st;
  const int64_t es = extent(blocks(rows), lds, blocks(cols), 4);
  if (rows_meet(w, ldw * ew, (int64_t)cols * ew, codes, ldc, cols, rows) ||
      bytes_meet(scales, es, w, extent(rows, ldw, cols, ew)) ||
      bytes_meet(scales, es, codes, extent(rows, ldc, cols, 1)))
    return fail(S2MOE_EINVAL, "%s: w, codes and scales overlap", fn);
  s2moe::QuantizeArgs a;
  a.n = rows;
  a.cols = cols;
  a.x = static_cast<const char*>(w);
  a.codes = static_cast<char*>(codes);
  a.scales = scales;
  a.ldx = ldw;
  a.ldc = ldc;
  a.lds = lds;
  a.x_type = w_dtype;
  return hip_status(fn, s2moe::launch_quantize_weight(a, static_cast<hipStream_t>(stream)));
}

s2moe_status s2moe_scaled_matmul(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                 const float* x_scales, int64_t ldxs, const void* w, int64_t ldw,
                                 const float* w_scales, int64_t ldws, void* out, int64_t ldo,
                                 int32_t out_dtype, void* stream) {
  const char* fn = "s2moe_scaled_matmul";
  s2moe_status st = check_count(fn, "m", m, 0, kMaxRows);
  if (st == S2MOE_OK) st = check_count(fn, "n", n, 1, kMaxRows);
  if (st == S2MOE_OK) st = check_cols(fn, "k", k, kMaxCols);
  if (st != S2MOE_OK) return st;
  if ((int64_t)m * n > (int64_t)1 << 34)
    return fail(S2MOE_EUNSUPPORTED, "%s: m n = %d %d exceeds 2^34", fn, m, n);
  if (!is_float(out_dtype))
    return fail(S2MOE_EINVAL, "%s: out_dtype = %d must be F32 or BF16", fn, out_dtype);
  if (m == 0) return ok();
  S2MOE_REQUIRE_PTR(x);
  S2MOE_REQUIRE_INTS(x_scales);
  S2MOE_REQUIRE_PTR(w);
  S2MOE_REQUIRE_INTS(w_scales);
  S2MOE_REQUIRE_PTR(out);
  if ((st = check_stride(fn, "ldx", ldx, k, 1)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldxs", ldxs, m, 0)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldw", ldw, k, 1)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldws", ldws, blocks(k), 0)) != S2MOE_OK) return st;
  if ((st = check_stride(fn, "ldo", ldo, n, 0)) != S2MOE_OK) return st;
  const int64_t eo = extent(m, ldo, n, elt(out_dtype));
  if (bytes_meet(out, eo, x, extent(m, ldx, k, 1)) || bytes_meet(out, eo, w, extent(n, ldw, k, 1)) ||
      bytes_meet(out, eo, x_scales, extent(blocks(k), ldxs, m, 4)) ||
      bytes_meet(out, eo, w_scales, extent(blocks(n), ldws, blocks(k), 4)))
    return fail(S2MOE_EINVAL, "%s: out overlaps an input", fn);
  s2moe::MatmulArgs a;
  a.m = m;
  a.n = n;
  a.k = k;
  a.x = static_cast<const uint8_t*>(x);
  a.xs = x_scales;
  a.w = static_cast<const uint8_t*>(w);
  a.ws = w_scales;
  a.out = static_cast<char*>(out);
  a.ldx = ldx;
  a.ldxs = ldxs;
  a.ldw = ldw;
  a.ldws = ldws;
  a.ldo = ldo;
  a.f32 = out_dtype == S2MOE_F32;
  return hip_status(fn, s2moe::launch_scaled_matmul(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
