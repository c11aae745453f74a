// Attention of drafted tokens over the paged cache.
//
// Rows.  The query heads of one kv head read the same keys, so the G = Hq / Hkv
// heads of a sequence's T nodes are T G rows of one product with the keys,
// taken 16 NT at a time by a workgroup.
//
// Products.  S^T = K Q^T and O^T = V^T P^T, so that a lane holds scores of one
// row: the maximum and the sum of a row need no exchange but over the four
// 16-lane groups, and the scores are, in the registers where the first product
// leaves them, the operand of the second.  That takes row m of the x-th of two
// 16-key tiles to be key 8 (m / 4) + 4 x + m % 4 of the step: lane group g then
// holds keys 8 g .. 8 g + 7, and the cache keeps eight neighbouring tokens of one
// coordinate of V together, so V is read in the order in which it is needed.
// No operand passes through LDS.
//
// Softmax.  One pass with a running maximum per row; it may lag behind the true
// one by 2^8, so that the accumulators are rescaled about once a row.
//
// Split.  The work is a list of units (sequence, kv head, row block, 128 keys),
// cut into equal stretches, one for each of a fixed number of workgroups,
// whatever the lengths are: the host does not know them.  Within a workgroup
// the four waves take 32 keys each.  A row block that one workgroup does not
// finish goes to the workspace in parts, and a second launch joins them.
#include "attention.h"
#include "attn_common.h"

namespace s2moe {
namespace {

#ifndef S2MOE_TREE_WIDE
#define S2MOE_TREE_WIDE 32
#endif
constexpr int kTile = 128;  // keys of a unit, 32 a wave

// A row block whose parts the joining launch adds, as the workgroup that has
// its first keys leaves it.
struct Split {
  int parts;  // 0: none starts here
  int slot;   // of this workgroup's part; the following workgroups' is their first
  int first;  // first token of the tree
  int head;   // kv head
  int row0;   // first row
  int rows;
};

template <typename E>
struct Type;
template <>
struct Type<uint16_t> {
  typedef bf16x8 frag;          // 8 of k
  static constexpr int kK = 8;  // elements of 16 bytes
};
template <>
struct Type<float> {
  typedef f32x4 frag;
  static constexpr int kK = 4;
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Four products of one k step of 4 each: element j of the fragments.
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

template <typename E, int D, int NT>
struct TreePlan {
  static constexpr int kRows = 16 * NT;
  // Workgroups that fit a compute unit.
  static constexpr int kPerCu = NT == 2 && D * sizeof(E) == 512 ? 1 : 2;
  static constexpr int kGroups = 256 * kPerCu;
  static constexpr size_t kPartFloats = (size_t)kRows * (D + 2);
  static constexpr size_t kBytes = kGroups * (2 * kPartFloats * 4 + sizeof(Split));
};

__device__ __forceinline__ bool sane(const TreeArgs& a, int first, int end) {
  return first >= 0 && first < end && end <= a.n_tokens;
}

// Tree and context of request i: first token, nodes, cached tokens, table row.
struct Request {
  int first, T, len, total;
  const int32_t* row;
};
__device__ __forceinline__ Request request(const TreeArgs& a, int i) {
  Request r{};
  r.first = constant(a.tok_off, i);
  const int end = constant(a.tok_off, i + 1), s = constant(a.seqs, i);
  if (!sane(a, r.first, end) || s < 0 || s >= a.max_seqs) return r;
  r.T = min(end - r.first, a.max_nodes);
  const int cap = a.max_pages << a.log_p;
  r.len = min(max(constant(a.length, s), 0), cap);
  r.total = r.len + min(r.T, cap - r.len);
  r.row = a.table + (int64_t)s * a.max_pages;
  return r;
}

// Ancestors of every node of a tree by pointer doubling: word 0 of a row of
// kMaskRow is all ones (cached tokens), 1 .. 8 the node's own bit and its
// ancestors', the rest zeros.  Nodes that hang below an invalid parent get
// dead_s != 0.
constexpr int kMaskRow = 11;
__device__ void ancestors(const int32_t* parent, int T, uint32_t* mask_s, int* jump_s,
                          uint8_t* dead_s) {
  const int i = threadIdx.x;
  int jump = -1, dead = 0;
  uint32_t word[kMaxNodes / 32];
#pragma unroll
  for (int x = 0; x < kMaxNodes / 32; ++x) word[x] = 0;
  if (i < T) {
    const int p = parent[i];
    dead = p != -1 && (p < 0 || p >= i);
    jump = dead ? -1 : p;
#pragma unroll
    for (int x = 0; x < kMaxNodes / 32; ++x) word[x] = x == i >> 5 ? 1u << (i & 31) : 0u;
    mask_s[i * kMaskRow] = ~0u;
    mask_s[i * kMaskRow + 9] = 0;
    mask_s[i * kMaskRow + 10] = 0;
  }
  for (;;) {
    if (i < T) {
#pragma unroll
      for (int x = 0; x < kMaxNodes / 32; ++x) mask_s[i * kMaskRow + 1 + x] = word[x];
      jump_s[i] = jump;
      dead_s[i] = dead;
    }
    if (!__syncthreads_or(jump >= 0)) break;
    if (jump >= 0) {
#pragma unroll
      for (int x = 0; x < kMaxNodes / 32; ++x) word[x] |= mask_s[jump * kMaskRow + 1 + x];
      dead |= dead_s[jump];
      jump = jump_s[jump];
    }
    __syncthreads();
  }
}

// Units before each request into before_s[0 .. n]; returns their number.
__device__ int64_t count_units(const TreeArgs& a, int RB, int64_t* before_s) {
  __shared__ int64_t wave_s[4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int64_t mine = 0;
  for (int x = 0; x < 4; ++x) {
    const int i = 4 * tid + x;
    if (i < a.n) {
      const Request r = request(a, i);
      before_s[i] = mine;
      mine += (int64_t)((r.T * a.G + RB - 1) / RB) * a.Hkv * ((r.total + kTile - 1) / kTile);
    }
  }
  int64_t inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  if (lane == 63) wave_s[w] = inc;
  __syncthreads();
  int64_t at = inc - mine, total = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    at += x < w ? wave_s[x] : 0;
    total += wave_s[x];
  }
  for (int x = 0; x < 4; ++x)
    if (4 * tid + x < a.n) before_s[4 * tid + x] += at;
  if (tid == 0) before_s[a.n] = total;
  __syncthreads();
  return total;
}

// The request that unit u falls into.
__device__ int request_of(int64_t u, int n, const int64_t* before_s) {
  int i = 0, hi = n;
  while (hi - i > 1) {
    const int mid = (i + hi) / 2;
    if (before_s[mid] <= u) i = mid; else hi = mid;
  }
  return i;
}

// Which of eight slots from node k0 on a row sees, k0 < 0 being cached tokens.
__device__ __forceinline__ uint32_t seen8(const uint32_t* mask, int k0) {
  k0 = min(max(k0, -32), kMaxNodes);
  const int x = (k0 + 32) >> 5;
  const uint64_t two = (uint64_t)mask[x + 1] << 32 | mask[x];
  return (uint32_t)(two >> (k0 & 31)) & 0xFFu;
}

__device__ __forceinline__ float largest(f32x4 a, f32x4 b) {
  return fmaxf(max3(max3(a[0], a[1], a[2]), a[3], b[0]), max3(b[1], b[2], b[3]));
}

// Scores of keys key .. key + 7 that a row does not see become -inf.
template <int NT>
__device__ __forceinline__ void mask_scores(f32x4 (&S)[2][NT], const int (&tok)[NT], const uint32_t* mask_s,
                                            int key, int len, int total) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const uint32_t seen = seen8(mask_s + tok[nt] * kMaskRow, key - len);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(seen >> e & 1) || key + e >= total) S[e >> 2][nt][e & 3] = -INFINITY;
  }
}

// Rows with a score past their limit move their maximum to it (m: the lane's
// largest scores).
template <int MT, int NT>
__device__ __forceinline__ void raise(const float (&m)[NT], float (&shift)[NT], float (&limit)[NT],
                                      float (&l)[NT], f32x4 (&O)[MT][NT]) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float top = max_groups(m[nt]);
    const bool moves = top > limit[nt], fresh = limit[nt] == -INFINITY;
    const float f = moves && !fresh ? exp2_fast(shift[nt] - top) : 1.f;
    shift[nt] = moves ? top : shift[nt];
    limit[nt] = moves ? top + kLag : limit[nt];
    l[nt] *= f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) O[mt][nt] *= f;
  }
}

// D / 16 elements of an output row, times `inv`; zeros where inv is 0.
template <typename E, int D>
__device__ __forceinline__ void write_row(const TreeArgs& a, int first, int hk, int row, int od,
                                          const float* o, float inv) {
  const int64_t at = (int64_t)(first + row / a.G) * a.ldo + (hk * a.G + row % a.G) * D + od;
#pragma unroll
  for (int y = 0; y < D / 16; y += 4) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : o[y + e] * inv;
    if constexpr (sizeof(E) == 4)
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at + y) = v;
    else
      *reinterpret_cast<bf16x4*>(reinterpret_cast<uint16_t*>(a.out) + at + y) = __builtin_convertvector(v, bf16x4);
  }
}

template <typename E, int D, int NT>
__global__ __launch_bounds__(256, (TreePlan<E, D, NT>::kPerCu)) void tree_kernel(TreeArgs a) {
  typedef typename Type<E>::frag frag;
  typedef TreePlan<E, D, NT> Plan;
  constexpr bool kF32 = sizeof(E) == 4;
  constexpr int RB = 16 * NT, MT = D / 16, ES = sizeof(E);
  constexpr int KC = D * ES / 64;  // 64-byte pieces of a key, 16 bytes a lane
  constexpr int VC = ES / 2;       // 16-byte pieces of eight values
  __shared__ int64_t before_s[kKvMaxRequests + 1];
  __shared__ __attribute__((aligned(16))) float sum_s[4][16][D + 4];
  __shared__ float m_s[4][RB], l_s[4][RB];
  __shared__ uint32_t mask_s[kMaxNodes * kMaskRow];
  __shared__ int jump_s[kMaxNodes];
  __shared__ uint8_t dead_s[kMaxNodes];

  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int n16 = lane & 15, g = lane >> 4;
  Split* const splits = reinterpret_cast<Split*>(a.ws + (size_t)Plan::kGroups * 2 * Plan::kPartFloats);
  float* const parts = a.ws;

  const int64_t total = count_units(a, RB, before_s);
  const int64_t share = (total + Plan::kGroups - 1) / Plan::kGroups;
  int64_t u = blockIdx.x * share;
  const int64_t u_end = min(u + share, total), u_first = u;
  int split_parts = 0;  // of a row block that starts here and goes on elsewhere

  int i = u < u_end ? request_of(u, a.n, before_s) : 0;
  const float c = a.scale * 1.44269504088896340736f;
  const int64_t head_bytes = (int64_t)a.P * D * ES, page_bytes = head_bytes * a.Hkv;
  // This lane's place in a half step of 16 keys, of the x-th key tile.
  const int k_lane = (8 * ((n16 >> 2) & 1) + (n16 & 3)) * D * ES + 16 * g;
  const int v_lane = ((g & 1) * D + n16) * 8 * ES;

  while (u < u_end) {
    i = __builtin_amdgcn_readfirstlane(i);
    while (before_s[i + 1] <= u) ++i;
    const Request r = request(a, i);
    const int tiles = (r.total + kTile - 1) / kTile, R = r.T * a.G, blocks = (R + RB - 1) / RB;
    const int64_t in = u - before_s[i];
    const int job = __builtin_amdgcn_readfirstlane((int)(in / tiles));
    const int t0 = __builtin_amdgcn_readfirstlane((int)(in - (int64_t)job * tiles));
    const int t1 = (int)min((int64_t)tiles, t0 + (u_end - u));
    const int hk = job / blocks, row0 = (job % blocks) * RB;
    const bool tail = t1 * kTile > r.len;
    if (tail) ancestors(a.parent + r.first, r.T, mask_s, jump_s, dead_s);

    int tok[NT];
    frag q[KC][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = min(row0 + 16 * nt + n16, R - 1);
      tok[nt] = row / a.G;
      const char* p = a.q + ((int64_t)(r.first + tok[nt]) * a.ldq + (hk * a.G + row % a.G) * D) * ES + 16 * g;
#pragma unroll
      for (int x = 0; x < KC; ++x) q[x][nt] = *reinterpret_cast<const frag*>(p + 64 * x);
    }

    f32x4 O[MT][NT];
    float shift[NT], limit[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      shift[nt] = 0.f;
      limit[nt] = -INFINITY;
      l[nt] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) O[mt][nt] = f32x4{};
    }
    frag K[2][KC], V[MT][VC];
    const char* const kb = a.k + hk * head_bytes + k_lane;
    const char* const vb = a.v + hk * head_bytes + v_lane;
    // Where the two half steps of 16 keys of tile t lie in the pools.
    const auto place = [&](int t, int64_t(&at)[2]) {
      const int key = t * kTile + 32 * w;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int slot = key + 16 * x;
        int page = constant(r.row, min(slot >> a.log_p, a.max_pages - 1));
        page = min(max(page, 0), a.n_pages - 1);
        at[x] = page * page_bytes + (int64_t)(slot & (a.P - 1)) * (D * ES);
      }
    };
    const auto load_k = [&](const int64_t(&at)[2]) {
      const char* p = kb + (n16 >> 3 ? at[1] : at[0]);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < KC; ++y) K[x][y] = *reinterpret_cast<const frag*>(p + 4 * x * D * ES + 64 * y);
    };
    const auto load_v = [&](const int64_t(&at)[2]) {
      const char* p = vb + (g >> 1 ? at[1] : at[0]);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int y = 0; y < VC; ++y) V[mt][y] = *reinterpret_cast<const frag*>(p + (16 * mt * 8) * ES + 16 * y);
    };

    int64_t now[2];
    place(t0, now);
    load_k(now);
    load_v(now);
    for (int t = t0; t < t1; ++t) {
      const int key0 = t * kTile + 32 * w;
      const bool more = t + 1 < t1;
      int64_t next[2];
      if (more) place(t + 1, next);
      f32x4 S[2][NT];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          S[x][nt] = f32x4{};
#pragma unroll
          for (int y = 0; y < KC; ++y) S[x][nt] = mma(K[x][y], q[y][nt], S[x][nt]);
        }
      if (more) load_k(next);
      const bool masked = key0 + 32 > r.len;
      if (masked) mask_scores<NT>(S, tok, mask_s, key0 + 8 * g, r.len, r.total);
      float m[NT];
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m[nt] = largest(S[0][nt], S[1][nt]) * c;
        over |= m[nt] > limit[nt];
      }
      if (__any(over)) raise<MT, NT>(m, shift, limit, l, O);
      float p[NT][8];
      frag P[NT][VC];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[nt][e] = exp2_fast(fmaf(S[e >> 2][nt][e & 3], c, -shift[nt]));
          l[nt] += p[nt][e];
        }
        if constexpr (kF32) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) P[nt][y][e] = p[nt][4 * y + e];
        } else {
          P[nt][0] = pack8(p[nt]);
        }
      }
      if (masked) {
        // A weight of zero does not hide an infinity or NaN: such values count
        // as zero, and where a weight meets one the row's sum becomes NaN.
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          bool bad = false;
#pragma unroll
          for (int y = 0; y < VC; ++y) bad |= any_nonfinite(V[mt][y]);
          if (__any(bad)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              f32x4 met = {};
#pragma unroll
              for (int y = 0; y < VC; ++y) met = mma(nonfinite_ones(V[mt][y]), P[nt][y], met);
#pragma unroll
              for (int e = 0; e < 4; ++e) O[mt][nt][e] = met[e] != 0.f ? NAN : O[mt][nt][e];
            }
#pragma unroll
            for (int y = 0; y < VC; ++y) V[mt][y] = finite_only(V[mt][y]);
          }
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int y = 0; y < VC; ++y) O[mt][nt] = mma(V[mt][y], P[nt][y], O[mt][nt]);
      if (more) load_v(next);
    }

    // The four waves' sums, by the largest maximum.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = sum_groups(l[nt]);
      if (g == 0) {
        m_s[w][16 * nt + n16] = limit[nt] == -INFINITY ? -INFINITY : shift[nt];
        l_s[w][16 * nt + n16] = l[nt];
      }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == tiles;
    const int slot = u == u_first ? 0 : 1;
    float* const part = parts + (2 * (size_t)blockIdx.x + slot) * Plan::kPartFloats;
    const int orow = tid >> 4, od = (tid & 15) * (D / 16);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (row0 + 16 * nt >= R) break;
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < 4; ++x) top = fmaxf(top, m_s[x][16 * nt + n16]);
      const float own = m_s[w][16 * nt + n16];
      const float f = own == -INFINITY ? 0.f : exp2_fast(own - top);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        *reinterpret_cast<f32x4*>(&sum_s[w][n16][16 * mt + 4 * g]) = O[mt][nt] * f;
      __syncthreads();
      const int row = row0 + 16 * nt + orow;
      if (row < R) {
        float om = -INFINITY, sum = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) om = fmaxf(om, m_s[x][16 * nt + orow]);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float mx = m_s[x][16 * nt + orow];
          sum += l_s[x][16 * nt + orow] * (mx == -INFINITY ? 0.f : exp2_fast(mx - om));
        }
        const bool dead = tail && dead_s[row / a.G];
        float o[D / 16];
#pragma unroll
        for (int y = 0; y < D / 64; ++y) {
          f32x4 v = *reinterpret_cast<const f32x4*>(&sum_s[0][orow][od + 4 * y]);
#pragma unroll
          for (int x = 1; x < 4; ++x) v += *reinterpret_cast<const f32x4*>(&sum_s[x][orow][od + 4 * y]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[4 * y + e] = v[e];
        }
        if (whole) {
          write_row<E, D>(a, r.first, hk, row, od, o, dead || sum == 0.f ? 0.f : 1.f / sum);
        } else {
          float* to = part + (16 * nt + orow) * (D + 2);
#pragma unroll
          for (int y = 0; y < D / 16; y += 2) *reinterpret_cast<f32x2*>(to + od + y) = f32x2{o[y], o[y + 1]};
          if ((tid & 15) == 0) *reinterpret_cast<f32x2*>(to + D) = f32x2{om, dead ? -1.f : sum};
        }
      }
      __syncthreads();
    }
    if (t0 == 0 && !whole) {
      const int64_t end = u + tiles;  // of the row block
      split_parts = (int)((end - 1) / share) - (int)blockIdx.x + 1;
      if (tid == 0)
        splits[blockIdx.x] = Split{split_parts, slot, r.first, hk, row0, min(RB, R - row0)};
    }
    u += t1 - t0;
  }
  if (split_parts == 0 && tid == 0) splits[blockIdx.x].parts = 0;
}

// Larger trees (bf16): rows are split over the waves, 16 NT each, and the keys and
// values of a stage are fetched once for all of them, by loads that go from the
// pages into LDS without a register between: three stages are in flight while one
// is used.  A wave fetches an eighth or quarter of a stage that lies in one page.
template <int D, int NT>
struct WidePlan {
  static constexpr int kRows = 64 * NT;
  static constexpr int kKeys = D == 128 ? 32 : 64;  // of a stage
  static constexpr int kStage = kKeys * D * 2;      // bytes of its keys, or values
  static constexpr int kRing = 4 * 2 * kStage;
  static constexpr int kPerCu = D == 128 && NT == 4 ? 1 : 2;
  static constexpr int kGroups = 256 * kPerCu;
  static constexpr size_t kPartFloats = (size_t)kRows * (D + 2);
  static constexpr size_t kBytes = kGroups * (2 * kPartFloats * 4 + sizeof(Split));
  static size_t lds(int n, int max_nodes) {
    return kRing + (size_t)(n + 1) * 8 + (size_t)max_nodes * (kMaskRow * 4 + 4 + 4);
  }
};

template <int D, int NT>
__global__ __launch_bounds__(256, (WidePlan<D, NT>::kPerCu)) void tree_wide_kernel(TreeArgs a) {
  typedef WidePlan<D, NT> Plan;
  constexpr int RB = Plan::kRows, MT = D / 16, KC = D / 32, SK = Plan::kKeys;
  constexpr int kLoads = Plan::kStage / 4096;  // 1 KB loads a wave makes for keys, or values
  constexpr int CH = D / 8;                    // 16-byte chunks of a key
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* const k_lds = smem;
  char* const v_lds = smem + 4 * Plan::kStage;
  int64_t* const before_s = reinterpret_cast<int64_t*>(smem + Plan::kRing);
  uint32_t* const mask_s = reinterpret_cast<uint32_t*>(before_s + a.n + 1);
  int* const jump_s = reinterpret_cast<int*>(mask_s + a.max_nodes * kMaskRow);
  uint8_t* const dead_s = reinterpret_cast<uint8_t*>(jump_s + a.max_nodes);

  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int n16 = lane & 15, g = lane >> 4;
  Split* const splits = reinterpret_cast<Split*>(a.ws + (size_t)Plan::kGroups * 2 * Plan::kPartFloats);
  const int64_t total = count_units(a, RB, before_s);
  const int64_t share = (total + Plan::kGroups - 1) / Plan::kGroups;
  int64_t u = blockIdx.x * share;
  const int64_t u_end = min(u + share, total), u_first = u;
  int split_parts = 0;
  int i = u < u_end ? request_of(u, a.n, before_s) : 0;
  const float c = a.scale * 1.44269504088896340736f;
  const int64_t head_bytes = (int64_t)a.P * D * 2, page_bytes = head_bytes * a.Hkv;

  // Chunk x of key r of a stage lies at chunk x ^ swizzle(r); values lie as they do
  // in the page.
  const auto swizzle = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
  uint32_t k_off[kLoads];
#pragma unroll
  for (int x = 0; x < kLoads; ++x) {
    const int r = x * (64 / CH) + lane / CH;  // within the wave's keys
    k_off[x] = r * D * 2 + (((lane % CH) ^ swizzle(w * (SK / 4) + r)) << 4);
  }
  const int key_row = 8 * (n16 >> 2) + (n16 & 3);  // of the first 16-key tile; the second's is 4 on

  while (u < u_end) {
    i = __builtin_amdgcn_readfirstlane(i);
    while (before_s[i + 1] <= u) ++i;
    const Request r = request(a, i);
    const int tiles = (r.total + kTile - 1) / kTile, R = r.T * a.G, blocks = (R + RB - 1) / RB;
    const int64_t in = u - before_s[i];
    const int job = __builtin_amdgcn_readfirstlane((int)(in / tiles));
    const int t0 = __builtin_amdgcn_readfirstlane((int)(in - (int64_t)job * tiles));
    const int t1 = (int)min((int64_t)tiles, t0 + (u_end - u));
    const int hk = job / blocks, row0 = (job % blocks) * RB;
    const int s0 = t0 * (kTile / SK), s1 = min(t1 * (kTile / SK), (r.total + SK - 1) / SK);
    const bool tail = t1 * kTile > r.len;
    const int wrow0 = row0 + 16 * NT * w;
    const bool active = wrow0 < R;

    // Stage s into its place in the ring; past the stretch, its last again.
    const char* const kb = a.k + hk * head_bytes;
    const char* const vb = a.v + hk * head_bytes;
    const auto page_of = [&](int s) {
      const int key = min(s, s1 - 1) * SK + w * (SK / 4);
      const int page = constant(r.row, min(key >> a.log_p, a.max_pages - 1));
      return min(max(page, 0), a.n_pages - 1);
    };
    const auto load_stage = [&](int s, int page) {
      const int key = min(s, s1 - 1) * SK + w * (SK / 4);
      const int64_t at = page * page_bytes + (int64_t)(key & (a.P - 1)) * (D * 2);
#pragma unroll
      for (int x = 0; x < kLoads; ++x)
        load_to_lds(kb + at, k_off[x], k_lds + (s & 3) * Plan::kStage + (w * kLoads + x) * 1024);
#pragma unroll
      for (int x = 0; x < kLoads; ++x)
        load_to_lds(vb + at, x * 1024 + lane * 16, v_lds + (s & 3) * Plan::kStage + (w * kLoads + x) * 1024);
    };
    load_stage(s0, page_of(s0));
    load_stage(s0 + 1, page_of(s0 + 1));
    load_stage(s0 + 2, page_of(s0 + 2));
    int page = page_of(s0 + 3);
    if (tail) ancestors(a.parent + r.first, r.T, mask_s, jump_s, dead_s);

    int tok[NT];
    bf16x8 q[KC][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = min(wrow0 + 16 * nt + n16, R - 1);
      tok[nt] = row / a.G;
      const char* p = a.q + ((int64_t)(r.first + tok[nt]) * a.ldq + (hk * a.G + row % a.G) * D) * 2 + 16 * g;
#pragma unroll
      for (int x = 0; x < KC; ++x) q[x][nt] = *reinterpret_cast<const bf16x8*>(p + 64 * x);
    }
    f32x4 O[MT][NT];
    float shift[NT], limit[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      shift[nt] = 0.f;
      limit[nt] = -INFINITY;
      l[nt] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) O[mt][nt] = f32x4{};
    }
    for (int s = s0; s < s1; ++s) {
      // Stage s is there for everybody, and stage s - 1, whose place stage s + 3
      // takes, is read by nobody any more.
      wait_loads<4 * kLoads>();
      __builtin_amdgcn_s_barrier();
      load_stage(s + 3, page);
      page = page_of(s + 4);
      if (!active) continue;
#pragma unroll
      for (int sub = 0; sub < SK / 32; ++sub) {
        const int key0 = s * SK + 32 * sub;
        const char* kt = k_lds + (s & 3) * Plan::kStage + 32 * sub * D * 2;
        const char* vt = v_lds + (s & 3) * Plan::kStage + (4 * sub + g) * (D * 16) + n16 * 16;
        f32x4 S[2][NT];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) S[x][nt] = f32x4{};
          const int row = key_row + 4 * x;
#pragma unroll
          for (int y = 0; y < KC; ++y) {
            const bf16x8 k = *reinterpret_cast<const bf16x8*>(kt + row * D * 2 + (((4 * y + g) ^ swizzle(row)) << 4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[x][nt] = mma(k, q[y][nt], S[x][nt]);
          }
        }
        const bool masked = key0 + 32 > r.len;
        if (masked) mask_scores<NT>(S, tok, mask_s, key0 + 8 * g, r.len, r.total);
        float m[NT];
        bool over = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          m[nt] = largest(S[0][nt], S[1][nt]) * c;
          over |= m[nt] > limit[nt];
        }
        if (__any(over)) raise<MT, NT>(m, shift, limit, l, O);
        bf16x8 P[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = exp2_fast(fmaf(S[e >> 2][nt][e & 3], c, -shift[nt]));
            l[nt] += p[e];
          }
          P[nt] = pack8(p);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          bf16x8 v = *reinterpret_cast<const bf16x8*>(vt + mt * 256);
          if (masked && __any(any_nonfinite(v))) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const f32x4 met = mma(nonfinite_ones(v), P[nt], f32x4{});
#pragma unroll
              for (int e = 0; e < 4; ++e) O[mt][nt][e] = met[e] != 0.f ? NAN : O[mt][nt][e];
            }
            v = finite_only(v);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) O[mt][nt] = mma(v, P[nt], O[mt][nt]);
        }
      }
    }
    wait_loads<0>();  // what was loaded past the stretch
    __syncthreads();  // nobody reads this stretch's stages or masks any more

    const bool whole = t0 == 0 && t1 == tiles;
    const int slot = u == u_first ? 0 : 1;
    float* const part = a.ws + (2 * (size_t)blockIdx.x + slot) * Plan::kPartFloats;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = wrow0 + 16 * nt + n16;
      const float sum = sum_groups(l[nt]);
      if (row >= R) continue;
      const bool dead = tail && dead_s[row / a.G];
      if (whole) {
        const float inv = dead || sum == 0.f ? 0.f : 1.f / sum;
        uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + (int64_t)(r.first + row / a.G) * a.ldo +
                      (hk * a.G + row % a.G) * D + 4 * g;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : O[mt][nt][e] * inv;
          *reinterpret_cast<bf16x4*>(o + 16 * mt) = __builtin_convertvector(v, bf16x4);
        }
      } else {
        float* to = part + (row - row0) * (D + 2);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 4; e += 2)
            *reinterpret_cast<f32x2*>(to + 16 * mt + 4 * g + e) = f32x2{O[mt][nt][e], O[mt][nt][e + 1]};
        if (g == 0)
          *reinterpret_cast<f32x2*>(to + D) = f32x2{limit[nt] == -INFINITY ? -INFINITY : shift[nt], dead ? -1.f : sum};
      }
    }
    if (t0 == 0 && !whole) {
      split_parts = (int)((u + tiles - 1) / share) - (int)blockIdx.x + 1;
      if (tid == 0)
        splits[blockIdx.x] = Split{split_parts, slot, r.first, hk, row0, min(RB, R - row0)};
    }
    u += t1 - t0;
    __syncthreads();  // dead_s is free again
  }
  if (split_parts == 0 && tid == 0) splits[blockIdx.x].parts = 0;
}

// Adds the parts of the row block that starts in workgroup blockIdx.x's stretch
// and ends in a later one's; blockIdx.y four rows, a wave every fourth part.
template <typename E, int D, typename Plan>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  __shared__ float m_s[4][4], l_s[4][4], o_s[4][4][D];
  const Split sp = reinterpret_cast<const Split*>(a.ws + (size_t)Plan::kGroups * 2 * Plan::kPartFloats)[blockIdx.x];
  const int row4 = blockIdx.y * 4;
  if (sp.parts == 0 || row4 >= sp.rows) return;
  const int tid = threadIdx.x, w = wave_id(), lr = (tid & 63) >> 4, od = (tid & 15) * (D / 16);
  const int row = min(row4 + lr, sp.rows - 1);
  float m = -INFINITY, l = 0.f, o[D / 16];
  bool dead = false;  // a sum of -1 marks a node that sees nothing
#pragma unroll
  for (int y = 0; y < D / 16; ++y) o[y] = 0.f;
#pragma unroll 2
  for (int p = w; p < sp.parts; p += 4) {
    const size_t slot = 2 * (size_t)(blockIdx.x + p) + (p == 0 ? sp.slot : 0);
    const float* from = a.ws + slot * Plan::kPartFloats + row * (D + 2);
    const f32x2 ml = *reinterpret_cast<const f32x2*>(from + D);
    dead |= ml[1] == -1.f;
    const float top = fmaxf(m, ml[0]);
    const float f = m == top ? 1.f : exp2_fast(m - top), h = ml[0] == top ? 1.f : exp2_fast(ml[0] - top);
    m = top;
    l = l * f + ml[1] * h;
#pragma unroll
    for (int y = 0; y < D / 16; y += 2) {
      const f32x2 v = *reinterpret_cast<const f32x2*>(from + od + y);
      o[y] = o[y] * f + v[0] * h;
      o[y + 1] = o[y + 1] * f + v[1] * h;
    }
  }
  if ((tid & 15) == 0) {
    m_s[w][lr] = m;
    l_s[w][lr] = dead ? -1.f : l;
  }
#pragma unroll
  for (int y = 0; y < D / 16; ++y) o_s[w][lr][od + y] = o[y];
  __syncthreads();
  if (w != 0 || row4 + lr >= sp.rows) return;
  float top = -INFINITY, sum = 0.f, f[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) top = fmaxf(top, m_s[x][lr]);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    f[x] = m_s[x][lr] == top ? 1.f : exp2_fast(m_s[x][lr] - top);
    dead |= l_s[x][lr] == -1.f;
    sum += l_s[x][lr] * f[x];
  }
#pragma unroll
  for (int y = 0; y < D / 16; ++y) {
    o[y] = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) o[y] += o_s[x][lr][od + y] * f[x];
  }
  write_row<E, D>(a, sp.first, sp.head, sp.row0 + row, od, o, dead || sum == 0.f ? 0.f : 1.f / sum);
}

template <typename E, int D, typename Plan>
hipError_t launch_join(const TreeArgs& a, hipStream_t s) {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  tree_join_kernel<E, D, Plan><<<dim3(Plan::kGroups, Plan::kRows / 4), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename E, int D, int NT>
struct ByKeys {  // waves split the keys
  static size_t bytes() { return TreePlan<E, D, NT>::kBytes; }
  static hipError_t launch(const TreeArgs& a, hipStream_t s) {
    tree_kernel<E, D, NT><<<TreePlan<E, D, NT>::kGroups, 256, 0, s>>>(a);
    return launch_join<E, D, TreePlan<E, D, NT>>(a, s);
  }
};

template <int D, int NT>
struct ByRows {  // waves split the rows
  typedef WidePlan<D, NT> Plan;
  static size_t bytes() { return Plan::kBytes; }
  static hipError_t launch(const TreeArgs& a, hipStream_t s) {
    static const hipError_t ready = hipFuncSetAttribute(
        reinterpret_cast<const void*>(tree_wide_kernel<D, NT>),
        hipFuncAttributeMaxDynamicSharedMemorySize, (int)Plan::lds(kKvMaxRequests, kMaxNodes));
    if (ready != hipSuccess) return ready;
    tree_wide_kernel<D, NT><<<Plan::kGroups, 256, Plan::lds(a.n, a.max_nodes), s>>>(a);
    return launch_join<uint16_t, D, Plan>(a, s);
  }
};

template <int D, typename F>
auto choose(int64_t rows, bool f32, F f) {
  if (f32) return rows <= 16 ? f(ByKeys<float, D, 1>{}) : f(ByKeys<float, D, 2>{});
  if (rows <= 16) return f(ByKeys<uint16_t, D, 1>{});
  if (rows <= S2MOE_TREE_WIDE) return f(ByKeys<uint16_t, D, 2>{});
  if (rows <= 64) return f(ByRows<D, 1>{});
  if (rows <= 128 || D == 128) return f(ByRows<D, 2>{});
  return f(ByRows<D, 4>{});
}

template <typename F>
auto choose(int G, int D, bool f32, int max_nodes, F f) {
  const int64_t rows = (int64_t)G * max_nodes;
  return D == 64 ? choose<64>(rows, f32, f) : choose<128>(rows, f32, f);
}

}  // namespace

size_t tree_attention_workspace(int Hq, int Hkv, int D, bool f32, int, int max_nodes) {
  return choose(Hq / Hkv, D, f32, max_nodes, [](auto k) { return decltype(k)::bytes(); });
}

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t s) {
  return choose(a.G, a.D, a.f32, a.max_nodes, [&](auto k) { return decltype(k)::launch(a, s); });
}

}  // namespace s2moe
