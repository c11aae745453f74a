// Positions of new tokens, and queries and keys rotated by them on the keys' way into
// the cache.
//
// A token of position p has, of each head, pairs of coordinates (a, b), and pair j turns
// by p f_j:  a' = a cos - b sin, b' = b cos + a sin.  The turn is p f_j / 2 pi in 64 bits,
// of which the nearest whole number is taken off before it is rounded to 32, so that far
// positions keep their angle, and angles next to a whole turn their small sine; sine, cosine
// and the products are fp32, and each element is rounded once.
//
// Bound: memory for prompts (17000 tokens, 32 query heads, 4 of keys and values, 128
// wide: 61 us, 5.5 TB/s, a large copy 5.2; 67 with queries through the caches, 65 and 71
// with their loads or stores so, 63 with keys and values past them too), latency for a
// step's few tokens (4.5 us).  Angles are worked out from the frequencies, a token's pairs by as many lanes, and
// shared through LDS: a table of them would have to be read.
#include <type_traits>

#include "attention.h"
#include "attn_common.h"

namespace s2moe {
namespace {

__device__ __forceinline__ bool in_range(int x, int n) { return x >= 0 && x < n; }

// Rows of request i, inside the packed tokens.
__device__ __forceinline__ void rows_of(const int32_t* tok_off, int i, int n_tokens, int* begin, int* end) {
  *begin = min(max(tok_off[i], 0), n_tokens);
  *end = min(max(tok_off[i + 1], *begin), n_tokens);
}

// Latency is all it costs: 2.2 us, with parents 2.6 to 4 (trees of up to 64 nodes).
// blockIdx.x a request.  Without parents blockIdx.y strides over its tokens.  With them
// 256 nodes are looked at at a time: `up` is each node's nearest ancestor that is not
// counted yet, and every step passes twice as many of them.
__global__ __launch_bounds__(256) void positions_kernel(KvCache c, int n_tokens, const int32_t* __restrict__ seqs,
                                                        const int32_t* __restrict__ tok_off,
                                                        const int32_t* __restrict__ parent, int32_t* pos) {
  __shared__ int up_s[256], depth_s[256];
  int begin, end;
  rows_of(tok_off, blockIdx.x, n_tokens, &begin, &end);
  const int s = seqs[blockIdx.x], me = threadIdx.x;
  const int first = in_range(s, c.max_seqs) ? c.length[s] : 0;
  if (parent == nullptr) {
    for (int i = begin + blockIdx.y * 256 + me; i < end; i += gridDim.y * 256)
      pos[i] = (int32_t)((uint32_t)first + (uint32_t)(i - begin));
    return;
  }
  for (int i0 = begin; i0 < end; i0 += 256) {
    const int i = i0 + me, node = i - begin;
    int up = -1, depth = 0;
    if (i < end) {
      const int p = parent[i];
      if (p >= 0 && p < node) {
        up = p - (i0 - begin);
        depth = 1;
        // An ancestor of an earlier round, whose depth is known.
        if (up < 0) depth = 1 + (int)((uint32_t)pos[begin + p] - (uint32_t)first);
      }
    }
    while (__syncthreads_or(up >= 0)) {
      up_s[me] = up;
      depth_s[me] = depth;
      __syncthreads();
      if (up >= 0) {
        depth += depth_s[up];
        up = up_s[up];
      }
    }
    if (i < end) pos[i] = (int32_t)((uint32_t)first + (uint32_t)depth);
    __syncthreads();  // what this round has written is read by the next one's
  }
}

constexpr int kPairs = 64;  // of a head, at most

// Elements of type E as 16 bytes: eight bf16 or four fp32.
template <typename E>
constexpr int kPer = 16 / (int)sizeof(E);

// A duo is two pieces of 16 bytes of a head that turn together: the pairs
// kPer duo .. kPer duo + kPer - 1, or elements that do not turn.  Pairs of neighbours lie
// in two neighbouring pieces; pairs of halves rot / 2 elements apart, and the duos of what
// does not turn after them.
template <typename E>
__device__ __forceinline__ int2 pieces_of(int duo, int rot, bool neighbours) {
  const int turned = rot / (2 * kPer<E>);
  return neighbours || duo >= turned ? int2{2 * duo, 2 * duo + 1} : int2{duo, duo + turned};
}

template <typename E>
__device__ __forceinline__ float element(u32x4 p, int i) {
  if constexpr (sizeof(E) == 4) return __uint_as_float(p[i]);
  else return __uint_as_float(i & 1 ? p[i / 2] & 0xFFFF0000u : p[i / 2] << 16);
}

// (x, y) turned by the kPer angles whose cosines and sines are at `cs`.
template <typename E>
__device__ __forceinline__ void turn(u32x4& x, u32x4& y, const float2* cs, bool neighbours) {
  constexpr int N = kPer<E>;
  float a[N], b[N], c[N], d[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // Pair i: neighbours are elements 2 i and 2 i + 1 of both pieces together.
    a[i] = element<E>(i < N / 2 ? x : y, 2 * i % N);
    b[i] = element<E>(i < N / 2 ? x : y, 2 * i % N + 1);
    c[i] = neighbours ? a[i] : element<E>(x, i);
    d[i] = neighbours ? b[i] : element<E>(y, i);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 t = cs[i];
    a[i] = c[i] * t.x - d[i] * t.y;
    b[i] = d[i] * t.x + c[i] * t.y;
  }
  float first[N], second[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    first[i] = neighbours ? (i & 1 ? b[i / 2] : a[i / 2]) : a[i];
    second[i] = neighbours ? (i & 1 ? b[(N + i) / 2] : a[(N + i) / 2]) : b[i];
  }
  if constexpr (sizeof(E) == 4) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = __float_as_uint(first[i]);
      y[i] = __float_as_uint(second[i]);
    }
  } else {
    x = __builtin_bit_cast(u32x4, pack8(first));
    y = __builtin_bit_cast(u32x4, pack8(second));
  }
}

__device__ __forceinline__ float2 cos_sin(int pos, float freq) {
  const double turns = (double)pos * (double)freq * 0.15915494309189535;  // 1 / 2 pi
  float s, c;
  sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
  return float2{c, s};
}

// The first workgroups: new tokens' keys and values, as the append of the cache does it, for
// every kv_parts-th kv head.  A wave has TW tokens.  With more than one the first token of a
// request and every token whose slot begins a group of eight write their group's; one goes
// alone.  The angles of a group are worked out once for all the wave's heads.  The others: the queries, a wave one token and
// every q_parts-th load of its heads.
template <typename E, int D, int TW>
__global__ __launch_bounds__(256) void append_rotated_kernel(KvCache c, RotateArgs a, int kv_blocks, int kv_parts, int q_parts) {
  constexpr int N = kPer<E>, kPieces = D / N, kDuos = kPieces / 2, VD = D / 64;
  typedef E E8 __attribute__((ext_vector_type(8)));
  typedef E EV __attribute__((ext_vector_type(VD)));
  // Rows two pairs longer than the pairs, so that tokens start in different banks.
  __shared__ __attribute__((aligned(16))) float2 cs_s[4][8][kPairs + 2];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = a.rot / 2, turned = half / N;
  const bool neighbours = a.neighbours;
  float2(*const cs)[kPairs + 2] = cs_s[wave];
  if ((int)blockIdx.x >= kv_blocks) {
    const int block = blockIdx.x - kv_blocks, part = block % q_parts, t = block / q_parts * 4 + wave;
    const int first = max(a.tok_off[0], 0), last = min(a.tok_off[a.n], a.n_tokens);
    if (t < first || t >= last) return;
    constexpr int kHeads = 64 / kDuos, kAtOnce = 4;  // of a load
    const int duo = lane % kDuos, h0 = part * kHeads + lane / kDuos, step = q_parts * kHeads;
    const int2 at = pieces_of<E>(duo, a.rot, neighbours);
    const u32x4* q = reinterpret_cast<const u32x4*>(reinterpret_cast<const E*>(a.q) + t * a.ldq);
    u32x4* to = reinterpret_cast<u32x4*>(reinterpret_cast<E*>(a.q_out) + t * a.ldqo);
    u32x4 u[kAtOnce], v[kAtOnce];
    const auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int g = min(h + i * step, a.Hq - 1);
        u[i] = __builtin_nontemporal_load(q + g * kPieces + at.x);
        v[i] = __builtin_nontemporal_load(q + g * kPieces + at.y);
      }
    };
    load(h0);
    if (lane < half) cs[0][lane] = cos_sin(a.pos[t], a.freq[lane]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int h = h0; h < a.Hq; h += kAtOnce * step) {
      if (h != h0) load(h);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (duo < turned) turn<E>(u[i], v[i], cs[0] + duo * N, neighbours);
        if (h + i * step < a.Hq) {
          __builtin_nontemporal_store(u[i], to + (h + i * step) * kPieces + at.x);
          __builtin_nontemporal_store(v[i], to + (h + i * step) * kPieces + at.y);
        }
      }
    }
    return;
  }
  const int kv_part = blockIdx.x % kv_parts;
  const int t0 = (blockIdx.x / kv_parts * 4 + wave) * TW;
  // Requests that begin at or before each token; lane x goes on with token t0 + x.
  int began[TW] = {}, i = -1;
  for (int i0 = 0; i0 < a.n; i0 += 64) {
    const int off = i0 + lane < a.n ? a.tok_off[i0 + lane] : 0x7FFFFFFF;
#pragma unroll
    for (int x = 0; x < TW; ++x) began[x] += __popcll(__ballot(off <= t0 + x));
  }
#pragma unroll
  for (int x = 0; x < TW; ++x) i = lane == x ? began[x] - 1 : i;
  const int mine = t0 + lane;
  int page = -1, slot = 0, count = 0;
  if (i >= 0 && mine < a.n_tokens) {
    const int begin = a.tok_off[i], end = min(a.tok_off[i + 1], a.n_tokens), s = a.seqs[i];
    if (mine >= begin && mine < end) {
      const bool known = in_range(s, c.max_seqs);
      const int64_t at = (int64_t)(known ? c.length[s] : 0) + mine - begin, nth = at >> c.log_p;
      if (TW == 1 || mine == begin || (at & 7) == 0) {
        slot = (int)(at & (c.P - 1));
        count = TW == 1 ? 1 : min(8 - (slot & 7), end - mine);
        if (known && at >= 0 && nth < c.max_pages) {
          const int p = c.table[(int64_t)s * c.max_pages + nth];
          if (in_range(p, c.n_pages) && c.refs[p] == 1) page = p;
        }
      }
    }
  }
#pragma unroll 1
  for (int x = 0; x < TW; ++x) {
    const int to = __shfl(page, x), at = __shfl(slot, x), n = __shfl(count, x), t = t0 + x;
    if (n == 0 || (to < 0 && a.k_out == nullptr)) continue;
    for (int j = lane; j < n * half; j += 64) {
      const int e = j / half, f = j - e * half;
      cs[e][f] = cos_sin(a.pos[t + e], a.freq[f]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int h = kv_part; h < c.Hkv; h += kv_parts) {
      const int64_t head = a.layer * c.layer_bytes() + to * c.page_bytes() + h * c.head_bytes();
      u32x4* const kt = reinterpret_cast<u32x4*>(c.k + head) + at * kPieces;
#pragma unroll
      for (int y = 0; y < 8 * kDuos / 64 || y == 0; ++y) {
        const int unit = lane + 64 * y, e = unit / kDuos, duo = unit % kDuos;
        if (e >= n) continue;
        const int2 p = pieces_of<E>(duo, a.rot, neighbours);
        const u32x4* k = reinterpret_cast<const u32x4*>(reinterpret_cast<const E*>(a.k) + (t + e) * a.ldk + h * D);
        u32x4 u = k[p.x], w = k[p.y];
        if (duo < turned) turn<E>(u, w, cs[e] + duo * N, neighbours);
        if (a.k_out != nullptr) {
          u32x4* o = reinterpret_cast<u32x4*>(reinterpret_cast<E*>(a.k_out) + (t + e) * a.ldko + h * D);
          o[p.x] = u;
          o[p.y] = w;
        }
        if (to >= 0) {
          kt[e * kPieces + p.x] = u;
          kt[e * kPieces + p.y] = w;
        }
      }
      if (to < 0) continue;
      const E* v = reinterpret_cast<const E*>(a.v) + t * a.ldv + h * D + VD * lane;
      E* const vt = reinterpret_cast<E*>(c.v + head) + (at >> 3) * D * 8 + VD * lane * 8;
      if (n == 8) {
        EV z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = *reinterpret_cast<const EV*>(v + e * a.ldv);
#pragma unroll
        for (int d = 0; d < VD; ++d) {
          E8 o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = z[e][d];
          *reinterpret_cast<E8*>(vt + d * 8) = o;
        }
      } else {
        for (int e = 0; e < n; ++e) {
          const EV z = *reinterpret_cast<const EV*>(v + e * a.ldv);
#pragma unroll
          for (int d = 0; d < VD; ++d) vt[d * 8 + (at & 7) + e] = z[d];
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename E, int D>
void launch_rotated(const KvCache& c, const RotateArgs& a, hipStream_t s) {
  constexpr int kHeads = 64 / (D / kPer<E> / 2);  // of a query load
  // Few tokens go alone, a wave each and kv head; groups of eight share angles and write
  // their values whole.  us alone / in groups, 32 heads over 8 of 128: 8 requests of 8 4.4 / 6.5,
  // 32 of 16 6.9 / 7.3, 300 of 4 16.0 / 16.5, 1024 of 1 18.8 / 24.2, 1 of 1300 15.6 / 10.3, 8 of
  // 512 35 / 20.  Requests of eight and more cross over at 600 tokens already (64 of 16: 12.2 /
  // 8.7), single tokens never do.
  const bool few = a.n_tokens < 1200;
  const int most = (a.Hq + kHeads - 1) / kHeads;
  // With waves enough, two kv heads a wave and half of the query heads: 17000 tokens, 32 heads
  // over 4 of 128, take 63.4 us so, 67.0 with a kv head each, 63.9 with all four in one, 61.7
  // with all of the queries and 72.4 with a quarter; 8000, 64 heads over 8 of 64, 36.7, 40.1
  // with a kv head each and 36.7 with all of the queries; 3500, 32 over 4, 17.9 and 16.9.
  const int kv_parts = a.n_tokens < 4096 ? c.Hkv : (c.Hkv + 1) / 2, q_parts = few ? most : most < 2 ? most : 2;
  const int per = few ? 4 : 32, kv_blocks = (a.n_tokens + per - 1) / per * kv_parts;
  const int grid = kv_blocks + (a.n_tokens + 3) / 4 * q_parts;
  if (few) append_rotated_kernel<E, D, 1><<<grid, 256, 0, s>>>(c, a, kv_blocks, kv_parts, q_parts);
  else append_rotated_kernel<E, D, 8><<<grid, 256, 0, s>>>(c, a, kv_blocks, kv_parts, q_parts);
}

}  // namespace

hipError_t launch_append_rotated(const KvCache& c, const RotateArgs& a, hipStream_t s) {
  if (c.f32) {
    if (c.D == 64) launch_rotated<uint32_t, 64>(c, a, s);
    else launch_rotated<uint32_t, 128>(c, a, s);
  } else {
    if (c.D == 64) launch_rotated<uint16_t, 64>(c, a, s);
    else launch_rotated<uint16_t, 128>(c, a, s);
  }
  return hipGetLastError();
}

hipError_t launch_positions(const KvCache& c, int n, int n_tokens, const int32_t* seqs, const int32_t* tok_off,
                            const int32_t* parent, int32_t* pos, hipStream_t s) {
  const int parts = (n_tokens / n + 1023) / 1024;
  const dim3 grid(n, parent != nullptr || parts < 1 ? 1 : parts > 64 ? 64 : parts);
  positions_kernel<<<grid, 256, 0, s>>>(c, n_tokens, seqs, tok_off, parent, pos);
  return hipGetLastError();
}

}  // namespace s2moe
