// Attention of drafted tokens over the paged cache.
//
// Rows.  The query heads of one kv head read the same keys, so the G = Hq / Hkv
// heads of a sequence's T nodes are T G rows of one product with the keys,
// a block of them to a workgroup.
//
// Products.  S^T = K Q^T and O^T = V^T P^T, so that a lane holds scores of one
// row: the maximum and the sum of a row need no exchange but over the four
// 16-lane groups, and the scores are, in the registers where the first product
// leaves them, the operand of the second.  That takes row m of the x-th of two
// 16-key tiles to be key 8 (m / 4) + 4 x + m % 4 of the step: lane group g then
// holds keys 8 g .. 8 g + 7, and the cache keeps eight neighbouring tokens of one
// coordinate of V together, so V is read in the order in which it is needed.
//
// Softmax.  One pass with a running maximum per row; it may lag behind the true
// one by 2^8, so that the accumulators are rescaled about once a row.
//
// Split.  The work is a list of units (sequence, kv head, row block, 128 keys),
// cut into equal stretches, one for each of a fixed number of workgroups,
// whatever the lengths are: the host does not know them.  A row block that one
// workgroup does not finish goes to the workspace in parts, and a second launch joins
// them.
//
// In bf16 the weights enter the second product rounded to bf16 (its operands have one
// type); their sum is taken in fp32 before that.
//
// Bound: reading the keys and values (16 sequences of 8192 tokens, 32/8 heads of 128,
// one node each: 101 us, 5.3 TB/s; 256 of 2048: 5.8; a plain read stream reaches 6.9);
// of the two workgroups on a compute unit the older ends at 73 us, the younger at 89.
// Ragged trees of up to 72 rows (64 sequences, 110 us, 3.9 TB/s) by waiting: 80 % of the
// waves' time, the matrix cores have 7 % of the cycles.  With hundreds of rows a wave's
// products and weights take turns and two waves a SIMD overlap them only in part (64
// nodes over 65537 tokens, 64/8 heads of 64: 107-117 us, 0.61 PFLOP/s; vector units 44 %
// of the cycles, matrix cores 25 %).  A single short sequence by dependent loads
// (offsets, length, page, keys) and the second launch: 11 us for one node over 2047
// tokens, 6.9 + 2.7.  16 nodes over 4093 take 14.6 + 4.5: 264 units for 512 workgroups,
// so half of them have nothing, and the others walk their 128 keys in four stages with
// a barrier each and leave 64 rows of parts.
#include "attention.h"
#include "attn_common.h"

namespace s2moe {
namespace {

constexpr int kTile = 128;  // keys of a unit

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

// 16 bytes along k, as the matrix instructions take them.
template <typename E>
struct Fragment {
  typedef bf16x8 type;
};
template <>
struct Fragment<float> {
  typedef f32x4 type;
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

// Where parts go: two for each workgroup, of as many rows as a row block can
// have, D sums, the maximum and the sum of weights each; then the splits.
struct Workspace {
  float* parts;
  Split* splits;
  int rows;
  __device__ __host__ Workspace(float* ws, int groups, int rows_, int D) : parts(ws), rows(rows_) {
    splits = reinterpret_cast<Split*>(ws + (size_t)groups * 2 * rows * (D + 2));
  }
  static size_t bytes(int groups, int rows, int D) {
    return groups * ((size_t)2 * rows * (D + 2) * 4 + sizeof(Split));
  }
  __device__ float* part(int group, int slot, int D) const {
    return parts + (2 * (size_t)group + slot) * rows * (D + 2);
  }
};
inline __device__ __host__ int part_rows(const TreeArgs& a, int RB) {
  const int64_t rows = (int64_t)a.G * a.max_nodes;
  return rows < RB ? (int)rows : RB;
}

// One request's tree and context: first token, nodes, cached tokens, those and
// the nodes' slots together, table row; and the units before it.
struct Request {
  int64_t before;
  int first, T, len, total, seq, pad;
};
__device__ __forceinline__ Request request(const TreeArgs& a, int i) {
  Request r{};
  r.first = a.tok_off[i];
  const int end = a.tok_off[i + 1];
  r.seq = a.seqs[i];
  const bool good = r.first >= 0 && r.first < end && end <= a.n_tokens && r.seq >= 0 && r.seq < a.max_seqs;
  r.T = good ? min(end - r.first, a.max_nodes) : 0;
  // No memory holds 2^31 tokens; below that tiles may be rounded up in 32 bits.
  const int cap = min(a.max_pages << a.log_p, 0x7FFFFF00);
  r.len = good ? min(max(a.length[r.seq], 0), cap) : 0;
  r.total = r.len + min(r.T, cap - r.len);
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

// Bytes of the requests, and of masks, parents and flags of a tree's nodes.
inline size_t shared_lists(int n, int max_nodes) {
  return (size_t)n * sizeof(Request) + (size_t)max_nodes * (kMaskRow * 4 + 4 + 4);
}

// All requests, with the units before each, into req_s[0 .. n - 1]; returns the
// number of units.  256 threads, ceil(n / 256) consecutive requests each.
__device__ int64_t list_requests(const TreeArgs& a, int RB, Request* req_s) {
  __shared__ int64_t wave_s[4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = (a.n + 255) >> 8;
  int64_t mine = 0;
  for (int x = 0; x < per; ++x) {
    const int i = per * tid + x;
    if (i >= a.n) break;
    Request r = request(a, i);
    r.before = mine;
    req_s[i] = r;
    mine += (int64_t)((r.T * a.G + RB - 1) / RB) * a.Hkv * ((r.total + kTile - 1) / kTile);
  }
  if (a.n == 1) {  // one thread knows all
    if (tid == 0) wave_s[0] = mine;
    __syncthreads();
    return wave_s[0];
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
  for (int x = 0; x < per; ++x)
    if (per * tid + x < a.n) req_s[per * tid + x].before += at;
  __syncthreads();
  return total;
}

// The last request that has units and whose first is at or before u.
__device__ int request_of(int64_t u, int n, const Request* req_s) {
  int i = 0, hi = n;
  while (hi - i > 1) {
    const int mid = (i + hi) / 2;
    if (req_s[mid].before <= u) i = mid; else hi = mid;
  }
  return __builtin_amdgcn_readfirstlane(i);
}

// The stretch of a row block that unit u starts: at most up to unit u_end.
struct Stretch {
  int first, T, len, total;      // as in Request
  const int32_t* row;            // of the table
  int R, hk, row0, t0, t1, tiles;
};
__device__ __forceinline__ Stretch stretch_of(const TreeArgs& a, const Request* req_s, int i, int RB,
                                              int64_t u, int64_t u_end) {
  const auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const Request r = req_s[i];
  Stretch z;
  z.first = same(r.first);
  z.T = same(r.T);
  z.len = same(r.len);
  z.total = same(r.total);
  z.row = a.table + (int64_t)same(r.seq) * a.max_pages;
  z.R = z.T * a.G;
  z.tiles = (z.total + kTile - 1) / kTile;
  const int in = same((int)(u - r.before)), blocks = (z.R + RB - 1) / RB;
  const int job = in / z.tiles;
  z.t0 = in - job * z.tiles;
  z.t1 = same((int)min((int64_t)z.tiles, z.t0 + (u_end - u)));
  z.hk = job / blocks;
  z.row0 = (job % blocks) * RB;
  return z;
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

// Where some rows do not see some keys: a weight of zero does not hide an infinity
// or NaN, so those values count as zero, and rows that see them get what they add up
// to.  Keys as in mask_scores.
template <int MT, int NT, int VC, typename frag>
__device__ __forceinline__ void hide_nonfinite(frag (&V)[MT][VC], const frag (&P)[NT][VC], f32x4 (&O)[MT][NT],
                                               const int (&tok)[NT], const uint32_t* mask_s, int key, int len, int total) {
  uint32_t bad = 0;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int y = 0; y < VC; ++y) bad |= any_nonfinite(V[mt][y]);
  if (__builtin_expect(!__any(bad != 0), 1)) return;
  uint32_t seen[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    seen[nt] = seen8(mask_s + tok[nt] * kMaskRow, key - len) & ((1u << min(max(total - key, 0), 8)) - 1);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      __builtin_amdgcn_sched_barrier(0);  // one after the other: registers
      f32x4 met = {};
#pragma unroll
      for (int y = 0; y < VC; ++y)
        met = mma(special_numbers(V[mt][y]), sight(seen[nt] >> (8 / VC * y), P[nt][y]), met);
#pragma unroll
      for (int e = 0; e < 4; ++e) O[mt][nt][e] += special_sum(met[e]);
    }
#pragma unroll
    for (int y = 0; y < VC; ++y) V[mt][y] = finite_only(V[mt][y]);
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

// Small trees: the four waves take 32 keys of a unit each, all rows of the block,
// and their sums are added at the end of a stretch.  No operand passes through
// LDS; the loads of the next unit are issued as soon as this one's registers are
// free, so that two workgroups a compute unit keep over 100 KB in flight.
template <typename E, int D, int NT>
struct KeysPlan {
  static constexpr int kRows = 16 * NT;
  // Workgroups that fit a compute unit.  fp32 at D = 128 needs all registers: with two
  // it spills, 16 sequences of 4096 tokens (32/8 heads) 103 -> 206 us at one node each,
  // 135 -> 307 at eight, one of 2047 12.8 -> 25.5.
  static constexpr int kPerCu = D * sizeof(E) == 512 ? 1 : 2;
  static constexpr int kGroups = 256 * kPerCu;
  static constexpr int kSums = 4 * 16 * (D + 4) * 4;  // bytes of the waves' sums of 16 rows
  static size_t lds(int n, int max_nodes) { return kSums + shared_lists(n, max_nodes); }
};

template <typename E, int D, int NT>
__global__ __launch_bounds__(256, (KeysPlan<E, D, NT>::kPerCu)) void tree_keys_kernel(TreeArgs a) {
  typedef typename Fragment<E>::type frag;
  typedef KeysPlan<E, D, NT> Plan;
  constexpr bool kF32 = sizeof(E) == 4;
  constexpr int RB = 16 * NT, MT = D / 16, ES = sizeof(E);
  constexpr int KC = D * ES / 64;  // 64-byte pieces of a key, 16 bytes a lane
  constexpr int VC = ES / 2;       // 16-byte pieces of eight values
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float(*const sum_s)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(smem);
  Request* const req_s = reinterpret_cast<Request*>(smem + Plan::kSums);
  uint32_t* const mask_s = reinterpret_cast<uint32_t*>(req_s + a.n);
  int* const jump_s = reinterpret_cast<int*>(mask_s + a.max_nodes * kMaskRow);
  uint8_t* const dead_s = reinterpret_cast<uint8_t*>(jump_s + a.max_nodes);
  __shared__ float m_s[4][RB], l_s[4][RB];

  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int n16 = lane & 15, g = lane >> 4;
  const Workspace ws(a.ws, Plan::kGroups, part_rows(a, RB), D);
  const int64_t total = list_requests(a, RB, req_s);
  const int64_t share = (total + Plan::kGroups - 1) / Plan::kGroups;
  int64_t u = blockIdx.x * share;
  const int64_t u_end = min(u + share, total), u_first = u;
  int split_parts = 0;  // of a row block that starts here and goes on elsewhere

  const float c = a.scale * 1.44269504088896340736f;
  const int64_t head_bytes = (int64_t)a.P * D * ES, page_bytes = head_bytes * a.Hkv;
  // This lane's place in a half step of 16 keys, of the x-th key tile.
  const int k_lane = (8 * ((n16 >> 2) & 1) + (n16 & 3)) * D * ES + 16 * g;
  const int v_lane = ((g & 1) * D + n16) * 8 * ES;

  while (u < u_end) {
    const Stretch r = stretch_of(a, req_s, request_of(u, a.n, req_s), RB, u, u_end);
    const int t0 = r.t0, t1 = r.t1, R = r.R, hk = r.hk, row0 = r.row0;
    const bool tail = t1 * kTile > r.len;

    int tok[NT];
    frag q[KC][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = min(row0 + 16 * nt + n16, R - 1);
      tok[nt] = row / a.G;
      const char* p = a.q + ((int64_t)(r.first + tok[nt]) * a.ldq + (hk * a.G + row - tok[nt] * a.G) * D) * ES + 16 * g;
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
    if (tail) ancestors(a.parent + r.first, r.T, mask_s, jump_s, dead_s);
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
      if (masked) hide_nonfinite<MT, NT, VC>(V, P, O, tok, mask_s, key0 + 8 * g, r.len, r.total);
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
    const bool whole = t0 == 0 && t1 == r.tiles;
    const int slot = u == u_first ? 0 : 1;
    float* const part = ws.part(blockIdx.x, slot, D);
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
      split_parts = (int)((u + r.tiles - 1) / share) - (int)blockIdx.x + 1;
      if (tid == 0)
        ws.splits[blockIdx.x] = Split{split_parts, slot, r.first, hk, row0, min(RB, R - row0)};
    }
    u += t1 - t0;
  }
  if (split_parts == 0 && tid == 0) ws.splits[blockIdx.x].parts = 0;
}

// Larger trees (bf16): the waves split the rows, 16 at a time in turn, and the keys
// and values of a stage are fetched once for all of them, by loads that go from the
// pages into LDS without a register between, three stages in flight while one is
// used (at D = 128 two of 64 keys each in place of four of 32: 108 -> 121 us for 64
// ragged trees).  A wave fetches a quarter of a stage, which lies in one page.
template <int D, int NT>
struct RowsPlan {
  static constexpr int kRows = 64 * NT;
  static constexpr int kKeys = D == 128 ? 32 : 64;  // of a stage
  static constexpr int kStage = kKeys * D * 2;      // bytes of its keys, or values
  static constexpr int kStages = 4;
  static constexpr int kRing = kStages * 2 * kStage;
  static constexpr int kGroups = 512;               // two fit a compute unit
  static size_t lds(int n, int max_nodes) {
    return kRing + shared_lists(n, max_nodes);
  }
};

template <int D>
struct RowsStage {  // what the waves of a workgroup share in a stretch
  char *k_lds, *v_lds;
  uint32_t* mask_s;
  uint8_t* dead_s;
  const char *kb, *vb;  // the head's keys and values in the first page
  int64_t page_bytes;
  uint32_t k_off[RowsPlan<D, 1>::kStage / 4096];
  int s0, s1;
};

// Stage s into its place in the ring; past the stretch, its last again.
template <int D>
__device__ __forceinline__ int rows_key(const RowsStage<D>& st, int s) {
  return min(s, st.s1 - 1) * RowsPlan<D, 1>::kKeys + wave_id() * (RowsPlan<D, 1>::kKeys / 4);
}
template <int D>
__device__ __forceinline__ int rows_page(const TreeArgs& a, const Stretch& r, const RowsStage<D>& st, int s) {
  const int page = constant(r.row, min(rows_key(st, s) >> a.log_p, a.max_pages - 1));
  return min(max(page, 0), a.n_pages - 1);
}
template <int D>
__device__ __forceinline__ void load_rows_stage(const TreeArgs& a, const Stretch& r, const RowsStage<D>& st, int s,
                                                int page) {
  typedef RowsPlan<D, 1> Plan;
  constexpr int kLoads = Plan::kStage / 4096;
  const int64_t at = page * st.page_bytes + (int64_t)(rows_key(st, s) & (a.P - 1)) * (D * 2);
  const int to = (s & (Plan::kStages - 1)) * Plan::kStage + wave_id() * kLoads * 1024;
#pragma unroll
  for (int x = 0; x < kLoads; ++x) load_to_lds(st.kb + at, st.k_off[x], st.k_lds + to + x * 1024);
#pragma unroll
  for (int x = 0; x < kLoads; ++x)
    load_to_lds(st.vb + at, x * 1024 + (threadIdx.x & 63) * 16, st.v_lds + to + x * 1024);
}

// A stretch, for a wave with NA tiles of 16 rows in it; all waves come through
// here with their own NA, and pass the same barriers.
template <int D, int NA>
__device__ __forceinline__ void rows_stretch(const TreeArgs& a, const Stretch& r, const RowsStage<D>& st, int page,
                                             bool tail, int tile0, bool whole, float* part) {
  typedef RowsPlan<D, 1> Plan;
  constexpr int MT = D / 16, KC = D / 32, SK = Plan::kKeys, kLoads = Plan::kStage / 4096;
  constexpr int N1 = NA > 0 ? NA : 1;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
  const auto swizzle = [](int x) { return D == 128 ? x & 15 : (x >> 1) & 7; };
  const int key_row = 8 * (n16 >> 2) + (n16 & 3);  // of the first 16-key tile; the second's is 4 on
  const float c = a.scale * 1.44269504088896340736f;
  int tok[N1];
  bf16x8 q[KC][N1];
  f32x4 O[MT][N1];
  float shift[N1], limit[N1], l[N1];
#pragma unroll
  for (int nt = 0; nt < NA; ++nt) {
    const int row = min(tile0 + 64 * nt + n16, r.R - 1);
    tok[nt] = row / a.G;
    const char* p = a.q + ((int64_t)(r.first + tok[nt]) * a.ldq + (r.hk * a.G + row - tok[nt] * a.G) * D) * 2 + 16 * g;
#pragma unroll
    for (int x = 0; x < KC; ++x) q[x][nt] = *reinterpret_cast<const bf16x8*>(p + 64 * x);
    shift[nt] = 0.f;
    limit[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) O[mt][nt] = f32x4{};
  }
  for (int s = st.s0; s < st.s1; ++s) {
    // Stage s is there for everybody, and the stage before, whose place is loaded
    // into, is read by nobody any more.
    wait_loads<(Plan::kStages - 2) * 2 * kLoads>();
    wait_lds();
    __builtin_amdgcn_s_barrier();
    load_rows_stage<D>(a, r, st, s + Plan::kStages - 1, page);
    page = rows_page<D>(a, r, st, s + Plan::kStages);
    if constexpr (NA > 0) {
      // 64 keys at a time as far as registers go: their products are independent.
      constexpr int NS = SK == 64 && NA <= 2 ? 2 : 1;
      const char* const kt = st.k_lds + (s & (Plan::kStages - 1)) * Plan::kStage;
      const char* const vt = st.v_lds + (s & (Plan::kStages - 1)) * Plan::kStage + g * (D * 16) + n16 * 16;
#pragma unroll
      for (int sub = 0; sub < SK / 32; sub += NS) {
        const int key0 = s * SK + 32 * sub;
        f32x4 S[NS][2][NA];
        bf16x8 V[NS][MT][1];
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int nt = 0; nt < NA; ++nt) S[z][x][nt] = f32x4{};
            const int row = 32 * (sub + z) + key_row + 4 * x;
#pragma unroll
            for (int y = 0; y < KC; ++y) {
              const bf16x8 k = *reinterpret_cast<const bf16x8*>(kt + row * D * 2 + (((4 * y + g) ^ swizzle(row)) << 4));
#pragma unroll
              for (int nt = 0; nt < NA; ++nt) S[z][x][nt] = mma(k, q[y][nt], S[z][x][nt]);
            }
          }
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            V[z][mt][0] = *reinterpret_cast<const bf16x8*>(vt + 4 * (sub + z) * (D * 16) + mt * 256);
        const bool masked = key0 + 32 * NS > r.len;
        if (masked)
#pragma unroll
          for (int z = 0; z < NS; ++z)
            mask_scores<NA>(S[z], tok, st.mask_s, key0 + 32 * z + 8 * g, r.len, r.total);
        float m[NA];
        bool over = false;
#pragma unroll
        for (int nt = 0; nt < NA; ++nt) {
          m[nt] = largest(S[0][0][nt], S[0][1][nt]);
          if (NS == 2) m[nt] = fmaxf(m[nt], largest(S[NS - 1][0][nt], S[NS - 1][1][nt]));
          m[nt] *= c;
          over |= m[nt] > limit[nt];
        }
        if (__any(over)) raise<MT, NA>(m, shift, limit, l, O);
        bf16x8 P[NS][NA][1];
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
          for (int nt = 0; nt < NA; ++nt) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              p[e] = exp2_fast(fmaf(S[z][e >> 2][nt][e & 3], c, -shift[nt]));
              l[nt] += p[e];
            }
            P[z][nt][0] = pack8(p);
          }
        if (masked)
#pragma unroll
          for (int z = 0; z < NS; ++z)
            hide_nonfinite<MT, NA, 1>(V[z], P[z], O, tok, st.mask_s, key0 + 32 * z + 8 * g, r.len, r.total);
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NA; ++nt) O[mt][nt] = mma(V[z][mt][0], P[z][nt][0], O[mt][nt]);
      }
    }
  }
  wait_loads<0>();  // what was loaded past the stretch
  __syncthreads();  // nobody reads this stretch's stages any more
#pragma unroll
  for (int nt = 0; nt < NA; ++nt) {
    const int row = tile0 + 64 * nt + n16;
    const float sum = sum_groups(l[nt]);
    if (row >= r.R) continue;
    const bool dead = tail && st.dead_s[tok[nt]];
    if (whole) {
      const float inv = dead || sum == 0.f ? 0.f : 1.f / sum;
      uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + (int64_t)(r.first + tok[nt]) * a.ldo +
                    (r.hk * a.G + row - tok[nt] * a.G) * D + 4 * g;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : O[mt][nt][e] * inv;
        *reinterpret_cast<bf16x4*>(o + 16 * mt) = __builtin_convertvector(v, bf16x4);
      }
    } else {
      float* to = part + (row - r.row0) * (D + 2);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
          *reinterpret_cast<f32x2*>(to + 16 * mt + 4 * g + e) = f32x2{O[mt][nt][e], O[mt][nt][e + 1]};
      if (g == 0)
        *reinterpret_cast<f32x2*>(to + D) = f32x2{limit[nt] == -INFINITY ? -INFINITY : shift[nt], dead ? -1.f : sum};
    }
  }
}

template <int D, int NT>
__global__ __launch_bounds__(256, 2) void tree_rows_kernel(TreeArgs a) {
  typedef RowsPlan<D, NT> Plan;
  constexpr int RB = Plan::kRows, SK = Plan::kKeys, kLoads = Plan::kStage / 4096, CH = D / 8;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Request* const req_s = reinterpret_cast<Request*>(smem + Plan::kRing);
  RowsStage<D> st;
  st.k_lds = smem;
  st.v_lds = smem + Plan::kStages * Plan::kStage;
  st.mask_s = reinterpret_cast<uint32_t*>(req_s + a.n);
  int* const jump_s = reinterpret_cast<int*>(st.mask_s + a.max_nodes * kMaskRow);
  st.dead_s = reinterpret_cast<uint8_t*>(jump_s + a.max_nodes);

  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const Workspace ws(a.ws, Plan::kGroups, part_rows(a, RB), D);
  const int64_t total = list_requests(a, RB, req_s);
  const int64_t share = (total + Plan::kGroups - 1) / Plan::kGroups;
  int64_t u = blockIdx.x * share;
  const int64_t u_end = min(u + share, total), u_first = u;
  int split_parts = 0;
  const int64_t head_bytes = (int64_t)a.P * D * 2;
  st.page_bytes = head_bytes * a.Hkv;
  // Chunk x of key i of a stage lies at chunk x ^ swizzle(i), so that reads spread
  // over all banks; values lie as they do in the page.
#pragma unroll
  for (int x = 0; x < kLoads; ++x) {
    const int i = x * (64 / CH) + lane / CH, at = w * (SK / 4) + i;  // within the wave's keys, the stage's
    st.k_off[x] = i * D * 2 + (((lane % CH) ^ (D == 128 ? at & 15 : (at >> 1) & 7)) << 4);
  }
  while (u < u_end) {
    const Stretch r = stretch_of(a, req_s, request_of(u, a.n, req_s), RB, u, u_end);
    st.kb = a.k + r.hk * head_bytes;
    st.vb = a.v + r.hk * head_bytes;
    st.s0 = r.t0 * (kTile / SK);
    st.s1 = min(r.t1 * (kTile / SK), (r.total + SK - 1) / SK);
    constexpr int kAhead = Plan::kStages - 1;
#pragma unroll
    for (int x = 0; x < kAhead; ++x) load_rows_stage<D>(a, r, st, st.s0 + x, rows_page<D>(a, r, st, st.s0 + x));
    const int page = rows_page<D>(a, r, st, st.s0 + kAhead);
    const bool tail = r.t1 * kTile > r.len, whole = r.t0 == 0 && r.t1 == r.tiles;
    if (tail) ancestors(a.parent + r.first, r.T, st.mask_s, jump_s, st.dead_s);
    const int slot = u == u_first ? 0 : 1;
    float* const part = ws.part(blockIdx.x, slot, D);
    const int tile0 = r.row0 + 16 * w;
    const int na = tile0 >= r.R ? 0 : min(NT, (r.R - tile0 + 63) / 64);
    if (na == 0) rows_stretch<D, 0>(a, r, st, page, tail, tile0, whole, part);
    else if (na == 1) rows_stretch<D, 1>(a, r, st, page, tail, tile0, whole, part);
    else if (NT == 2 || na == 2) rows_stretch<D, 2>(a, r, st, page, tail, tile0, whole, part);
    else rows_stretch<D, NT == 4 ? 4 : 0>(a, r, st, page, tail, tile0, whole, part);
    if (r.t0 == 0 && !whole) {
      split_parts = (int)((u + r.tiles - 1) / share) - (int)blockIdx.x + 1;
      if (tid == 0)
        ws.splits[blockIdx.x] = Split{split_parts, slot, r.first, r.hk, r.row0, min(RB, r.R - r.row0)};
    }
    u += r.t1 - r.t0;
    __syncthreads();  // dead_s is free again
  }
  if (split_parts == 0 && tid == 0) ws.splits[blockIdx.x].parts = 0;
}

// Adds the parts of a row block that several workgroups share; blockIdx.y four rows,
// a wave every W-th part.  blockIdx.x is the workgroup that has its first keys or
// (W = 8), where a call has few row blocks of many rows, the block's rank among the
// shared ones: then no workgroup comes for nothing, and each can have more waves.
template <typename E, int D, int W>
__global__ __launch_bounds__(64 * W) void tree_join_kernel(TreeArgs a, int groups, int RB) {
  __shared__ float m_s[W][4], l_s[W][4], o_s[W][4][D];
  const Workspace ws(a.ws, groups, part_rows(a, RB), D);
  int group = blockIdx.x;
  if constexpr (W == 8) {
    // groups <= 512: each thread looks at one.
    __shared__ int count_s[W], found_s;
    const uint64_t there = __ballot((int)threadIdx.x < groups && ws.splits[threadIdx.x].parts != 0);
    const int lane = threadIdx.x & 63, at = wave_id();
    if (lane == 0) count_s[at] = __popcll(there);
    if (threadIdx.x == 0) found_s = -1;
    __syncthreads();
    int before = 0;
    for (int x = 0; x < at; ++x) before += count_s[x];
    if ((there >> lane & 1) && before + __popcll(there & ((1ull << lane) - 1)) == (int)blockIdx.x)
      found_s = threadIdx.x;
    __syncthreads();
    group = __builtin_amdgcn_readfirstlane(found_s);
    if (group < 0) return;
  }
  const Split sp = ws.splits[group];
  const int row4 = blockIdx.y * 4;
  if (sp.parts == 0 || row4 >= sp.rows) return;
  const int tid = threadIdx.x, w = wave_id(), lr = (tid & 63) >> 4, od = (tid & 15) * (D / 16);
  const int row = min(row4 + lr, sp.rows - 1);
  float m = -INFINITY, l = 0.f, o[D / 16];
  bool dead = false;  // a sum of -1 marks a node that sees nothing
#pragma unroll
  for (int y = 0; y < D / 16; ++y) o[y] = 0.f;
#pragma unroll 4
  for (int p = w; p < sp.parts; p += W) {
    const float* from = ws.part(group + p, p == 0 ? sp.slot : 0, D) + row * (D + 2);
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
  float top = -INFINITY, sum = 0.f, f[W];
#pragma unroll
  for (int x = 0; x < W; ++x) top = fmaxf(top, m_s[x][lr]);
#pragma unroll
  for (int x = 0; x < W; ++x) {
    f[x] = m_s[x][lr] == top ? 1.f : exp2_fast(m_s[x][lr] - top);
    dead |= l_s[x][lr] == -1.f;
    sum += l_s[x][lr] * f[x];
  }
#pragma unroll
  for (int y = 0; y < D / 16; ++y) {
    o[y] = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) o[y] += o_s[x][lr][od + y] * f[x];
  }
  write_row<E, D>(a, sp.first, sp.head, sp.row0 + row, od, o, dead || sum == 0.f ? 0.f : 1.f / sum);
}

template <typename E, int D, typename Plan>
hipError_t launch_join(const TreeArgs& a, hipStream_t s) {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  static_assert(Plan::kGroups <= 512, "one thread a workgroup");
  const int rows = part_rows(a, Plan::kRows);
  const int64_t blocks = (int64_t)a.n * a.Hkv * (((int64_t)a.G * a.max_nodes + Plan::kRows - 1) / Plan::kRows);
  // Ranked, measured both ways for 1 to 64 sequences of 1000 to 65537 tokens and 1 to 64
  // nodes, six head layouts: where the rule ranks 0.63 to 1.06 times the other time,
  // mostly below 1 (one sequence of 16000, 32/4 heads of 128, 16 nodes 46 -> 29 us; 4 of
  // 2000, 32/8, 16 nodes 33 -> 22; 4 of 9000, 64 nodes 71 -> 74); where it does not 0.90
  // to 1.5 times, mostly above (16 of 1000, 64/8 heads of 64, 40 nodes 53 -> 79; 64 of
  // 1500, 32/4, one node 36 -> 37; but one of 16000, 32/4, one node 18.1 -> 16.4).
  if (rows > 16 && blocks < Plan::kGroups / 4)
    tree_join_kernel<E, D, 8><<<dim3((unsigned)blocks, (rows + 3) / 4), 512, 0, s>>>(a, Plan::kGroups, Plan::kRows);
  else
    tree_join_kernel<E, D, 4><<<dim3(Plan::kGroups, (rows + 3) / 4), 256, 0, s>>>(a, Plan::kGroups, Plan::kRows);
  return hipGetLastError();
}

template <typename E, int D_, int NT>
struct ByKeys {
  typedef KeysPlan<E, D_, NT> Plan;
  static constexpr int D = D_;
  static hipError_t launch(const TreeArgs& a, hipStream_t s) {
    static std::atomic<uint64_t> ready{0};
    const hipError_t err =
        allow_lds(reinterpret_cast<const void*>(tree_keys_kernel<E, D, NT>), Plan::lds(kKvMaxRequests, kMaxNodes), ready);
    if (err != hipSuccess) return err;
    tree_keys_kernel<E, D, NT><<<Plan::kGroups, 256, Plan::lds(a.n, a.max_nodes), s>>>(a);
    return launch_join<E, D, Plan>(a, s);
  }
};

template <int D_, int NT>
struct ByRows {
  typedef RowsPlan<D_, NT> Plan;
  static constexpr int D = D_;
  static hipError_t launch(const TreeArgs& a, hipStream_t s) {
    static std::atomic<uint64_t> ready{0};
    const hipError_t err =
        allow_lds(reinterpret_cast<const void*>(tree_rows_kernel<D, NT>), Plan::lds(kKvMaxRequests, kMaxNodes), ready);
    if (err != hipSuccess) return err;
    tree_rows_kernel<D, NT><<<Plan::kGroups, 256, Plan::lds(a.n, a.max_nodes), s>>>(a);
    return launch_join<uint16_t, D, Plan>(a, s);
  }
};

// The kernel by type, head size and the rows that the largest tree can have.  Up to 16
// rows the waves split the keys.  us by rows / by keys, 32/8 heads of 128: over 4096 tokens 4
// rows 11.2 / 11.5, 16 rows 14 / 15, 20 rows 13 / 17, 32 rows 14 / 18; 16 sequences of
// 8192 101 / 101, 106 / 105, 108 / 126, 113 / 129; 64 of up to 6000 163 / 156, 168 /
// 161, 175 / 198, 175 / 197.  fp32 goes by keys only.  The rows are those of max_nodes,
// since the host knows no other: one node a sequence announced as 16 takes 11.1 us for
// 10.3 (one of 2047 tokens), 14.6 for 12.5 (4 of 2000), 79 for 74 (64 of 1500).
template <int D, typename F>
auto choose(int64_t rows, bool f32, F f) {
  if (f32) return rows <= 16 ? f(ByKeys<float, D, 1>{}) : f(ByKeys<float, D, 2>{});
  return rows <= 16 ? f(ByKeys<uint16_t, D, 1>{}) : f(ByRows<D, D == 64 ? 4 : 2>{});
}

template <typename F>
auto choose(const TreeArgs& a, F f) {
  const int64_t rows = (int64_t)a.G * a.max_nodes;
  return a.D == 64 ? choose<64>(rows, a.f32, f) : choose<128>(rows, a.f32, f);
}

}  // namespace

size_t tree_attention_workspace(const TreeArgs& a) {
  return choose(a, [&](auto k) {
    typedef decltype(k) K;
    return Workspace::bytes(K::Plan::kGroups, part_rows(a, K::Plan::kRows), K::D);
  });
}

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t s) {
  return choose(a, [&](auto k) { return decltype(k)::launch(a, s); });
}

}  // namespace s2moe
