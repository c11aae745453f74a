// Page operations of the key / value cache and the write of new tokens.
//
// Nothing here computes: a page operation reads and writes some integers per
// sequence, and copies or moves tokens of every layer.  Integer work goes to
// one workgroup per request (fork, free, the end of commit) or to one
// workgroup for all of them (reserve, whose grants depend on each other);
// what they decide does not depend on timing: a free page is one that nobody
// holds, and the lowest ids are taken first, in the order of the requests.
//
// Bound: latency for the integer work (64 requests: fork, free and the end of commit
// 5 us each, reserve 11; where the only free pages are a pool's last, one workgroup
// reads all of refs twice: 22 us at 10 000 pages, 72 at 50 000, 42 with over 256
// requests and so 1024 threads), memory for the
// copies (the used slots of 16 pages of 64 tokens to four branches each, 24 layers, 8
// heads of 128, 239 MB written and 60 read: 69 us, 4.3 TB/s) and the move (up to 16
// accepted tokens of each branch over the same layers: 42 us, 2.2 TB/s) and
// for new tokens (about 17000, 8 heads of 128: 34 us where a large copy takes 28).
#include <type_traits>

#include "attention.h"
#include "common.h"

namespace s2moe {
namespace {

// Whether request i's id appears among the ids before it.  Block-wide.
__device__ bool repeated(const int32_t* __restrict__ ids, int i) {
  const int32_t id = ids[i];
  int hit = 0;
  for (int j = threadIdx.x; j < i; j += blockDim.x) hit |= ids[j] == id;
  return __syncthreads_or(hit);
}

__device__ __forceinline__ bool in_range(int x, int n) { return x >= 0 && x < n; }

__device__ __forceinline__ int pages_of(const KvCache& c, int64_t tokens) {
  const int64_t n = (tokens + c.P - 1) >> c.log_p;
  return n < 0 ? 0 : (n > c.max_pages ? c.max_pages : (int)n);
}

__global__ void kv_init_kernel(KvCache c) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = t; i < (int64_t)c.max_seqs * c.max_pages; i += step) c.table[i] = -1;
  for (int64_t i = t; i < c.max_seqs; i += step) c.length[i] = 0;
  for (int64_t i = t; i < c.n_pages; i += step) c.refs[i] = 0;
}

__global__ __launch_bounds__(256) void kv_fork_kernel(KvCache c, int n,
                                                      const int32_t* __restrict__ src,
                                                      const int32_t* __restrict__ dst,
                                                      int32_t* __restrict__ status) {
  const int i = blockIdx.x;
  const int a = src[i], b = dst[i];
  int hit = !in_range(a, c.max_seqs) || !in_range(b, c.max_seqs);
  for (int j = threadIdx.x; j < n; j += blockDim.x) hit |= dst[j] == a || (j < i && dst[j] == b);
  if (__syncthreads_or(hit)) {
    if (threadIdx.x == 0) status[i] = kKvBadSeq;
    return;
  }
  int32_t* to = c.table + (int64_t)b * c.max_pages;
  const int32_t* from = c.table + (int64_t)a * c.max_pages;
  const bool busy = c.length[b] != 0 || to[0] >= 0;
  __syncthreads();  // every thread has looked before any writes
  if (busy) {
    if (threadIdx.x == 0) status[i] = kKvBusy;
    return;
  }
  const int held = pages_of(c, c.length[a]);
  for (int j = threadIdx.x; j < held; j += blockDim.x) {
    const int p = from[j];
    if (!in_range(p, c.n_pages)) continue;
    to[j] = p;
    atomicAdd(&c.refs[p], 1);
  }
  if (threadIdx.x == 0) {
    c.length[b] = c.length[a];
    status[i] = 0;
  }
}

// Gives back the pages of table row `row` from index `first` on.
__device__ void drop_pages(const KvCache& c, int32_t* row, int first) {
  for (int j0 = first; j0 < c.max_pages; j0 += blockDim.x) {
    const int j = j0 + threadIdx.x;
    int end = 1;
    if (j < c.max_pages) {
      const int p = row[j];
      end = p < 0;
      if (p >= 0) {
        row[j] = -1;
        if (p < c.n_pages) atomicSub(&c.refs[p], 1);
      }
    }
    if (__syncthreads_or(end)) break;  // a row's pages lie together at its start
  }
}

__global__ __launch_bounds__(256) void kv_free_kernel(KvCache c, const int32_t* __restrict__ seqs,
                                                      int32_t* __restrict__ status) {
  const int i = blockIdx.x, s = seqs[i];
  const bool bad = repeated(seqs, i) || !in_range(s, c.max_seqs);
  if (threadIdx.x == 0) status[i] = bad ? kKvBadSeq : 0;
  if (bad) return;
  drop_pages(c, c.table + (int64_t)s * c.max_pages, 0);
  if (threadIdx.x == 0) c.length[s] = 0;
}

// Sum of x over the threads before this one; *total over all.
__device__ int64_t scan_block(int64_t x, int64_t* total, int64_t* waves) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  int64_t inc = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();  // `waves` is free again
  if (lane == 63) waves[w] = inc;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int j = 0; j < nw; ++j) {
    const int64_t y = waves[j];
    before += j < w ? y : 0;
    all += y;
  }
  *total = all;
  return before + inc - x;
}

// How many of ids[0 .. i - 1] (LDS, 16-byte aligned) equal x.
__device__ int count_before(const int* ids, int i, int x) {
  int n = 0;
  for (int j = 0; j < i; j += 4) {
    const int4 v = *reinterpret_cast<const int4*>(ids + j);
    n += (v.x == x) + (j + 1 < i && v.y == x) + (j + 2 < i && v.z == x) + (j + 3 < i && v.w == x);
  }
  return n;
}

// Grants of one reserve call: one workgroup, one thread per request.  A wave looks
// at 1024 pages a sweep, 64 at a time, so that the free ones come in order from
// ballots.
__global__ __launch_bounds__(1024) void kv_reserve_kernel(KvCache c, int n,
                                                          const int32_t* __restrict__ seqs,
                                                          const int32_t* __restrict__ extra,
                                                          int32_t* __restrict__ copied,
                                                          int32_t* __restrict__ status) {
  __shared__ __attribute__((aligned(16))) int seq_s[1024], shared_s[1024];
  __shared__ int first_s[1024], held_s[1024], copy_s[1024], to_s[1024], waves[16];
  __shared__ int64_t sums_s[16];
  const int i = threadIdx.x, lane = i & 63, w = i >> 6, nw = blockDim.x >> 6;
  const bool live = i < n;
  const int s = live ? seqs[i] : -1;
  const int more = live ? extra[i] : 0;
  seq_s[i] = s;
  to_s[i] = -1;
  int st = 0, need = 0, held = 0, page = -1, refs = 0;
  int64_t last = 0;
  int32_t* row = nullptr;
  if (live && !in_range(s, c.max_seqs)) st = kKvBadSeq;
  if (live && !st) {
    row = c.table + (int64_t)s * c.max_pages;
    const int64_t len = c.length[s], want = len + more;
    if (more < 0 || len < 0 || want > ((int64_t)c.max_pages << c.log_p)) {
      st = kKvTooLong;
    } else {
      const int target = pages_of(c, want);
      held = pages_of(c, len);
      last = len >> c.log_p;
      if (more > 0 && (len & (c.P - 1)) != 0) {
        const int p = row[last];
        if (in_range(p, c.n_pages)) {
          refs = c.refs[p];
          if (refs > 1) page = p;
        }
      }
      while (held < target && row[held] >= 0) ++held;
      need = target - held > 0 ? target - held : 0;
    }
  }
  __syncthreads();
  if (live && st != kKvBadSeq && count_before(seq_s, i, s) > 0) {
    st = kKvBadSeq;
    need = 0;
    page = -1;
  }
  shared_s[i] = page;
  __syncthreads();
  // Of the sequences that share a page the last keeps it, if the others get their copies.
  const int copy = page >= 0 && refs - count_before(shared_s, i, page) > 1;
  const int take = need + copy;
  // 1024 requests of up to 2^27 pages pass 32 bits; past the pool's pages all are alike.
  int64_t all;
  const int64_t first = scan_block(take, &all, sums_s);
  const int total = (int)min(all, (int64_t)c.n_pages + 1);
  first_s[i] = (int)min(first, (int64_t)c.n_pages + 1);
  held_s[i] = held;
  copy_s[i] = copy;
  // How many free pages there are, up to `total`; then who gets which.
  int free_pages = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = 0;
    const int stop = pass == 0 ? total : (total < free_pages ? total : free_pages);
    for (int64_t p0 = 0; p0 < c.n_pages && seen < stop; p0 += nw * 1024) {
      const int64_t mine = p0 + w * 1024 + lane;
      int r[16];
#pragma unroll
      for (int b = 0; b < 16; ++b) r[b] = mine + 64 * b < c.n_pages ? c.refs[mine + 64 * b] : 1;
      uint64_t free_mask[16];
      int here = 0;
#pragma unroll
      for (int b = 0; b < 16; ++b) {
        free_mask[b] = __ballot(r[b] == 0);
        here += __popcll(free_mask[b]);
      }
      __syncthreads();  // `waves` is free again
      if (lane == 0) waves[w] = here;
      __syncthreads();
      int f0 = seen;
      for (int j = 0; j < nw; ++j) {
        f0 += j < w ? waves[j] : 0;
        seen += waves[j];
      }
      if (pass == 0) continue;
#pragma unroll
      for (int b = 0; b < 16; ++b) {
        const int f = f0 + __popcll(free_mask[b] & ((1ull << lane) - 1));
        f0 += __popcll(free_mask[b]);
        if (r[b] != 0 || f >= stop) continue;
        const int p = (int)(mine + 64 * b);
        int lo = 0, hi = n;  // the last request whose first page is at or before f
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (first_s[mid] <= f) lo = mid; else hi = mid;
        }
        const int end = lo + 1 < n ? first_s[lo + 1] : total;
        if (end > free_pages) continue;  // its request is not granted
        const int k = f - first_s[lo];
        if (k < copy_s[lo])
          to_s[lo] = p;
        else
          c.table[(int64_t)seq_s[lo] * c.max_pages + held_s[lo] + k - copy_s[lo]] = p;
        c.refs[p] = 1;
      }
    }
    if (pass == 0) {
      free_pages = seen;
      __syncthreads();  // first_s and its like are complete
    }
  }
  bool refused = take > 0 && first + take > free_pages;
  if (total > free_pages) {
    // Who got no copy still holds the page: the last sharer cannot write to it either.
    shared_s[i] = refused && copy ? page : -1;
    __syncthreads();
    refused |= page >= 0 && !copy && count_before(shared_s, i, page) > 0;
  }
  __syncthreads();  // to_s is complete
  if (live) {
    if (refused) st = kKvNoPages;
    const int to = st ? -1 : to_s[i];
    if (to >= 0) {
      row[last] = to;
      atomicSub(&c.refs[page], 1);
    }
    copied[2 * i] = to >= 0 ? page : -1;
    copied[2 * i + 1] = to;
    status[i] = st;
  }
}

// The pages that a reserve call copies: blockIdx.y the request, blockIdx.x a
// (layer, head).  A head's part of a page is one stretch in both pools.
__global__ __launch_bounds__(256) void kv_copy_kernel(KvCache c, const int32_t* __restrict__ seqs,
                                                      const int32_t* __restrict__ copied) {
  const int i = blockIdx.y;
  const int from = copied[2 * i], to = copied[2 * i + 1];
  if (from < 0) return;
  const int used = ((c.length[seqs[i]] & (c.P - 1)) + 7) & ~7;
  const int l = blockIdx.x / c.Hkv, h = blockIdx.x % c.Hkv;
  const int64_t base = l * c.layer_bytes() + h * c.head_bytes();
  const int64_t a = base + from * c.page_bytes(), b = base + to * c.page_bytes();
  const int n16 = used * c.D * c.elt() / 16;
  for (int j = threadIdx.x; j < n16; j += blockDim.x) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(c.k + a + 16 * j);
    const u32x4 y = *reinterpret_cast<const u32x4*>(c.v + a + 16 * j);
    *reinterpret_cast<u32x4*>(c.k + b + 16 * j) = x;
    *reinterpret_cast<u32x4*>(c.v + b + 16 * j) = y;
  }
}

// Status of a commit request, the same in both launches.  Block-wide.  note(j, p,
// from, to): the accepted node of rank j is p, its slots' pages are from and to.
template <typename F>
__device__ int check_commit(const KvCache& c, int i, int max_path,
                            const int32_t* __restrict__ seqs, const int32_t* __restrict__ path,
                            int acc, F note) {
  const int s = seqs[i];
  int bad = 0;
  if (in_range(s, c.max_seqs) && acc >= 0 && (path == nullptr || acc <= max_path)) {
    const int64_t len = c.length[s];
    const int32_t* row = c.table + (int64_t)s * c.max_pages;
    // The page of a slot that the sequence holds alone; -1 where it does not.
    const auto alone = [&](int64_t pos) {
      const int64_t at = pos >> c.log_p;
      if (pos < 0 || at >= c.max_pages) return -1;
      const int page = row[at];
      return in_range(page, c.n_pages) && c.refs[page] == 1 ? page : -1;
    };
    if (path != nullptr) {
      for (int j = threadIdx.x; j < acc; j += blockDim.x) {
        const int p = path[(int64_t)i * max_path + j];
        const int before = j > 0 ? path[(int64_t)i * max_path + j - 1] : -1;
        const int from = alone(len + p), to = alone(len + j);
        bad |= p <= before || from < 0 || to < 0;
        note(j, p, from, to);
      }
    } else {
      for (int64_t j = threadIdx.x * (int64_t)c.P; j < acc; j += blockDim.x * (int64_t)c.P)
        bad |= alone(len + j) < 0;
      bad |= acc > 0 && alone(len + acc - 1) < 0;
    }
    bad |= len < 0;
  } else {
    bad = 1;
  }
  if (repeated(seqs, i) || !in_range(s, c.max_seqs)) return kKvBadSeq;
  return __syncthreads_or(bad) ? kKvBadPath : 0;
}

// Moves one request's accepted tokens, blockIdx.y the request, a wave one (layer,
// head).  path[j] >= j, so in ascending order nothing is overwritten that has yet to
// be read: a later token's source is at or after its own target, past what is written
// before.  Keys move 16 bytes a lane, 1 KB a load; of the values a lane has D / 64
// coordinates and puts together whole groups of eight tokens.
template <typename E, int D>
__global__ __launch_bounds__(256) void kv_move_kernel(KvCache c, int max_path,
                                                      const int32_t* __restrict__ seqs,
                                                      const int32_t* __restrict__ path,
                                                      const int32_t* __restrict__ n_accept) {
  constexpr int kPieces = D * (int)sizeof(E) / 16, kAtOnce = 64 / kPieces;  // of a key; keys a load
  constexpr int VD = D / 64;
  typedef E E8 __attribute__((ext_vector_type(8)));
  __shared__ int node_s[kMaxNodes], from_p[kMaxNodes], to_p[kMaxNodes];
  const int i = blockIdx.y, acc = n_accept[i];
  int stays = 0;
  if (check_commit(c, i, max_path, seqs, path, acc, [&](int j, int p, int from, int to) {
        node_s[j] = p;
        from_p[j] = from;
        to_p[j] = to;
        stays = p == j;
      }))
    return;
  const int j0 = __syncthreads_count(stays);  // path[j] == j for j < j0
  if (j0 == acc) return;
  const int len = c.length[seqs[i]], lane = threadIdx.x & 63;
  const int64_t page_bytes = c.page_bytes();
  const int piece = lane % kPieces, mine = lane / kPieces;
  const auto slot = [&](int node) { return (len + node) & (c.P - 1); };
  for (int lh = blockIdx.x * 4 + wave_id(); lh < c.L * c.Hkv; lh += gridDim.x * 4) {
    const int64_t base = (lh / c.Hkv) * c.layer_bytes() + (lh % c.Hkv) * c.head_bytes();
    int jb = j0, g0 = (len + j0) & ~7;
    while (jb < acc || g0 < len + acc) {  // up to 4 kAtOnce keys, and a group of values
      u32x4 x[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int j = jb + y * kAtOnce + mine;
        if (j < acc)
          x[y] = *reinterpret_cast<const u32x4*>(c.k + base + from_p[j] * page_bytes +
                                                 (slot(node_s[j]) * kPieces + piece) * 16);
      }
      const int j1 = g0 - len;  // the group's first slot as a node, below 0 for older tokens
      const bool group = g0 < len + acc;
      char* to = nullptr;
      E8 v[VD];
      E y8[VD][8];
      if (group) {
        to = c.v + base + to_p[max(j1, j0)] * page_bytes + (int64_t)(g0 & (c.P - 1)) * D * sizeof(E);
#pragma unroll
        for (int z = 0; z < VD; ++z) v[z] = *reinterpret_cast<const E8*>(to + (lane + 64 * z) * sizeof(E8));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = j1 + e;
          if (j >= j0 && j < acc) {
            const int from = slot(node_s[j]);
            const E* p = reinterpret_cast<const E*>(c.v + base + from_p[j] * page_bytes) + (from >> 3) * D * 8 + (from & 7);
#pragma unroll
            for (int z = 0; z < VD; ++z) y8[z][e] = p[(lane + 64 * z) * 8];
          }
        }
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int j = jb + y * kAtOnce + mine;
        if (j < acc)
          *reinterpret_cast<u32x4*>(c.k + base + to_p[j] * page_bytes + (slot(j) * kPieces + piece) * 16) = x[y];
      }
      if (group) {
#pragma unroll
        for (int z = 0; z < VD; ++z) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (j1 + e >= j0 && j1 + e < acc) v[z][e] = y8[z][e];
          *reinterpret_cast<E8*>(to + (lane + 64 * z) * sizeof(E8)) = v[z];
        }
      }
      jb += 4 * kAtOnce;
      g0 += 8;
    }
  }
}

__global__ __launch_bounds__(256) void kv_commit_kernel(KvCache c, int max_path,
                                                        const int32_t* __restrict__ seqs,
                                                        const int32_t* __restrict__ path,
                                                        const int32_t* __restrict__ n_accept,
                                                        int32_t* __restrict__ status) {
  const int i = blockIdx.x, acc = n_accept[i];
  const int st = check_commit(c, i, max_path, seqs, path, acc, [](int, int, int, int) {});
  if (threadIdx.x == 0) status[i] = st;
  if (st) return;
  const int s = seqs[i];
  const int64_t len = (int64_t)c.length[s] + acc;
  drop_pages(c, c.table + (int64_t)s * c.max_pages, pages_of(c, len));
  if (threadIdx.x == 0) c.length[s] = (int)len;
}

// New tokens of one layer: blockIdx.x 4 TW packed tokens, TW a wave, blockIdx.y a kv
// head.  The first token of a request and every token whose slot begins a group of
// eight write their group's tokens; the others have nothing to do.  The lanes look up
// the tokens' pages together; then one has D / 64 coordinates of the values, and a
// group that is whole goes out 16 bytes or more a coordinate.
template <typename E, int D, int TW>
__global__ __launch_bounds__(256) void kv_append_kernel(KvCache c, AppendArgs a) {
  constexpr int kPieces = D * (int)sizeof(E) / 16, VD = D / 64;
  typedef E E8 __attribute__((ext_vector_type(8)));
  typedef E EV __attribute__((ext_vector_type(VD)));
  const int lane = threadIdx.x & 63, t0 = (blockIdx.x * 4 + wave_id()) * TW, h = blockIdx.y;
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
    if (mine >= begin && mine < end && in_range(s, c.max_seqs)) {
      const int64_t pos = (int64_t)c.length[s] + mine - begin, at = pos >> c.log_p;
      if (pos >= 0 && at < c.max_pages && (mine == begin || (pos & 7) == 0)) {
        const int p = c.table[(int64_t)s * c.max_pages + at];
        if (in_range(p, c.n_pages) && c.refs[p] == 1) page = p;
        slot = (int)(pos & (c.P - 1));
        count = min(8 - (slot & 7), end - mine);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < TW; ++x) {
    const int to = __builtin_amdgcn_readlane(page, x), at = __builtin_amdgcn_readlane(slot, x);
    const int n = __builtin_amdgcn_readlane(count, x), t = t0 + x;
    if (to < 0) continue;
    const int64_t head = a.layer * c.layer_bytes() + to * c.page_bytes() + h * c.head_bytes();
    const E* k = reinterpret_cast<const E*>(a.k) + t * a.ldk + h * D;
    const E* v = reinterpret_cast<const E*>(a.v) + t * a.ldv + h * D + VD * lane;
    u32x4* const kt = reinterpret_cast<u32x4*>(c.k + head) + at * kPieces;
    E* const vt = reinterpret_cast<E*>(c.v + head) + (at >> 3) * D * 8 + VD * lane * 8;
    if (n == 8) {
      EV z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = *reinterpret_cast<const EV*>(v + e * a.ldv);
      u32x4 y[8 * kPieces / 64];
#pragma unroll
      for (int b = 0; b < 8 * kPieces / 64; ++b) {
        const int q = lane + 64 * b;
        y[b] = reinterpret_cast<const u32x4*>(k + (q / kPieces) * a.ldk)[q % kPieces];
      }
#pragma unroll
      for (int b = 0; b < 8 * kPieces / 64; ++b) kt[lane + 64 * b] = y[b];
#pragma unroll
      for (int d = 0; d < VD; ++d) {
        E8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = z[e][d];
        *reinterpret_cast<E8*>(vt + d * 8) = o;
      }
    } else {
      for (int q = lane; q < n * kPieces; q += 64)
        kt[q] = reinterpret_cast<const u32x4*>(k + (q / kPieces) * a.ldk)[q % kPieces];
      for (int e = 0; e < n; ++e) {
        const EV z = *reinterpret_cast<const EV*>(v + e * a.ldv);
#pragma unroll
        for (int d = 0; d < VD; ++d) vt[d * 8 + (at & 7) + e] = z[d];
      }
    }
  }
}

// f(element, head size) for the cache's type.
template <typename F>
void by_type(const KvCache& c, F f) {
  if (c.f32) {
    if (c.D == 64) f(uint32_t{}, std::integral_constant<int, 64>{});
    else f(uint32_t{}, std::integral_constant<int, 128>{});
  } else {
    if (c.D == 64) f(uint16_t{}, std::integral_constant<int, 64>{});
    else f(uint16_t{}, std::integral_constant<int, 128>{});
  }
}

}  // namespace

hipError_t launch_kv_init(const KvCache& c, hipStream_t s) {
  kv_init_kernel<<<256, 256, 0, s>>>(c);
  return hipGetLastError();
}

hipError_t launch_kv_fork(const KvCache& c, int n, const int32_t* src, const int32_t* dst,
                          int32_t* status, hipStream_t s) {
  kv_fork_kernel<<<n, 256, 0, s>>>(c, n, src, dst, status);
  return hipGetLastError();
}

hipError_t launch_kv_reserve(const KvCache& c, int n, const int32_t* seqs, const int32_t* extra,
                             int32_t* copied, int32_t* status, hipStream_t s) {
  kv_reserve_kernel<<<1, n <= 256 ? 256 : 1024, 0, s>>>(c, n, seqs, extra, copied, status);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  kv_copy_kernel<<<dim3(c.L * c.Hkv, n), 256, 0, s>>>(c, seqs, copied);
  return hipGetLastError();
}

hipError_t launch_kv_commit(const KvCache& c, int n, int max_path, const int32_t* seqs,
                            const int32_t* path, const int32_t* n_accept, int32_t* status,
                            hipStream_t s) {
  if (path != nullptr && max_path > 0) {
    // Four (layer, head) a workgroup, or more where that makes over 2048 workgroups.
    const int most = 2048 / n > 0 ? 2048 / n : 1, want = (c.L * c.Hkv + 3) / 4;
    const dim3 grid(want < most ? want : most, n);
    by_type(c, [&](auto e, auto d) {
      kv_move_kernel<decltype(e), decltype(d)::value><<<grid, 256, 0, s>>>(c, max_path, seqs, path, n_accept);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  kv_commit_kernel<<<n, 256, 0, s>>>(c, max_path, seqs, path, n_accept, status);
  return hipGetLastError();
}

hipError_t launch_kv_free(const KvCache& c, int n, const int32_t* seqs, int32_t* status,
                          hipStream_t s) {
  kv_free_kernel<<<n, 256, 0, s>>>(c, seqs, status);
  return hipGetLastError();
}

hipError_t launch_kv_append(const KvCache& c, const AppendArgs& a, hipStream_t s) {
  // A wave takes a token where requests bring few, else eight, of which about one
  // begins a group.  us at one / eight, 8 heads of 128: 48 requests of 1 token 5.3 / 6.8,
  // 16 of 6 5.5 / 6.6, 16 of 16 5.5 / 5.5, 5 of 3000 35 / 21.
  const bool few = a.n_tokens / a.n < 8;
  const int per = few ? 4 : 32;
  const dim3 grid((a.n_tokens + per - 1) / per, c.Hkv);
  by_type(c, [&](auto e, auto d) {
    typedef decltype(e) E;
    constexpr int D = decltype(d)::value;
    if (few)
      kv_append_kernel<E, D, 1><<<grid, 256, 0, s>>>(c, a);
    else
      kv_append_kernel<E, D, 8><<<grid, 256, 0, s>>>(c, a);
  });
  return hipGetLastError();
}

}  // namespace s2moe
