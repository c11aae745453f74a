// Page operations of the key / value cache and the write of new tokens.
//
// Nothing here computes: a page operation reads and writes some integers per
// sequence, and copies or moves tokens of every layer.  Integer work goes to
// one workgroup per request (fork, free, the end of commit) or to one
// workgroup for all of them (reserve, whose grants depend on each other);
// what they decide does not depend on timing: a free page is one that nobody
// holds, and the lowest ids are taken first, in the order of the requests.
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

// Sum of x over the threads before this one; *total over all.  1024 threads.
__device__ int scan_1024(int x, int* total, int* waves) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int inc = x;
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();  // `waves` is free again
  if (lane == 63) waves[w] = inc;
  __syncthreads();
  int before = 0, all = 0;
  for (int j = 0; j < 16; ++j) {
    const int y = waves[j];
    before += j < w ? y : 0;
    all += y;
  }
  *total = all;
  return before + inc - x;
}

// Grants of one reserve call, one thread per request.
__global__ __launch_bounds__(1024) void kv_reserve_kernel(KvCache c, int n,
                                                          const int32_t* __restrict__ seqs,
                                                          const int32_t* __restrict__ extra,
                                                          int32_t* __restrict__ copied,
                                                          int32_t* __restrict__ status) {
  __shared__ int seq_s[1024], shared_s[1024], first_s[1024], held_s[1024], copy_s[1024], to_s[1024],
      waves[16];
  const int i = threadIdx.x;
  const bool live = i < n;
  const int s = live ? seqs[i] : -1;
  seq_s[i] = s;
  __syncthreads();
  int st = 0, need = 0, held = 0, page = -1;
  int64_t last = 0;
  int32_t* row = nullptr;
  if (live) {
    if (!in_range(s, c.max_seqs)) st = kKvBadSeq;
    for (int j = 0; j < i && !st; ++j) st = seq_s[j] == s ? kKvBadSeq : 0;
  }
  if (live && !st) {
    row = c.table + (int64_t)s * c.max_pages;
    const int64_t len = c.length[s], want = len + extra[i];
    if (extra[i] < 0 || len < 0 || want > ((int64_t)c.max_pages << c.log_p)) {
      st = kKvTooLong;
    } else {
      const int target = pages_of(c, want);
      held = pages_of(c, len);
      while (held < target && row[held] >= 0) ++held;
      need = target - held > 0 ? target - held : 0;
      last = len >> c.log_p;
      if (extra[i] > 0 && (len & (c.P - 1)) != 0) {
        const int p = row[last];
        if (in_range(p, c.n_pages) && c.refs[p] > 1) page = p;
      }
    }
  }
  shared_s[i] = page;
  __syncthreads();
  // Of the sequences that share a page the last keeps it.
  int copy = 0;
  if (page >= 0) {
    int rank = 0;
    for (int j = 0; j < i; ++j) rank += shared_s[j] == page;
    copy = c.refs[page] - rank > 1;
  }
  const int take = need + copy;
  int total;
  const int first = scan_1024(take, &total, waves);
  first_s[i] = first;
  held_s[i] = held;
  copy_s[i] = copy;
  to_s[i] = -1;
  // How many free pages there are, up to `total`; then who gets which.
  int free_pages = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = 0;
    const int stop = pass == 0 ? total : (total < free_pages ? total : free_pages);
    for (int64_t p0 = 0; p0 < c.n_pages && seen < stop; p0 += 1024 * 16) {
      const int64_t mine = p0 + threadIdx.x * 16;
      uint32_t free_mask = 0;
      for (int b = 0; b < 16; ++b)
        if (mine + b < c.n_pages && c.refs[mine + b] == 0) free_mask |= 1u << b;
      int here;
      int f = seen + scan_1024(__popc(free_mask), &here, waves);
      if (pass == 1) {
        for (; free_mask != 0 && f < stop; free_mask &= free_mask - 1, ++f) {
          const int p = (int)(mine + __ffs(free_mask) - 1);
          int lo = 0, hi = n;  // the last request whose first page is at or before f
          while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first_s[mid] <= f) lo = mid; else hi = mid;
          }
          const int end = lo + 1 < n ? first_s[lo + 1] : total;
          if (end > free_pages) continue;  // its request is not granted
          int32_t* r = c.table + (int64_t)seq_s[lo] * c.max_pages;
          const int k = f - first_s[lo];
          if (k < copy_s[lo]) {
            to_s[lo] = p;
          } else {
            r[held_s[lo] + k - copy_s[lo]] = p;
          }
          c.refs[p] = 1;
        }
      }
      seen += here;
    }
    if (pass == 0) free_pages = seen;
  }
  __syncthreads();  // to_s[] is complete
  if (live) {
    if (take > 0 && first + take > free_pages) st = kKvNoPages;
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

// Status of a commit request, the same in both launches.  Block-wide.
__device__ int check_commit(const KvCache& c, int i, int max_path,
                            const int32_t* __restrict__ seqs, const int32_t* __restrict__ path,
                            int acc) {
  const int s = seqs[i];
  if (repeated(seqs, i) || !in_range(s, c.max_seqs)) return kKvBadSeq;
  const int64_t len = c.length[s];
  if (len < 0 || acc < 0 || (path != nullptr && acc > max_path)) return kKvBadPath;
  int bad = 0;
  const int32_t* row = c.table + (int64_t)s * c.max_pages;
  // Every slot that is kept lies in a page that the sequence holds alone.
  const auto alone = [&](int64_t pos) {
    const int64_t at = pos >> c.log_p;
    if (at >= c.max_pages) return false;
    const int page = row[at];
    return in_range(page, c.n_pages) && c.refs[page] == 1;
  };
  if (path != nullptr) {
    for (int j = threadIdx.x; j < acc; j += blockDim.x) {
      const int p = path[(int64_t)i * max_path + j];
      const int before = j > 0 ? path[(int64_t)i * max_path + j - 1] : -1;
      bad |= p <= before || !alone(len + p) || !alone(len + j);
    }
  } else {
    for (int64_t j = threadIdx.x * (int64_t)c.P; j < acc; j += blockDim.x * (int64_t)c.P)
      bad |= !alone(len + j);
    bad |= acc > 0 && !alone(len + acc - 1);
  }
  return __syncthreads_or(bad) ? kKvBadPath : 0;
}

// Moves one request's accepted tokens, blockIdx.y the request.  A thread
// keeps to one 16-byte piece of a key, or one coordinate of the values, of
// one (layer, head), and moves it for the path's nodes in ascending order:
// path[j] >= j, so what it overwrites it has read before.
template <typename E>
__global__ __launch_bounds__(256) void kv_move_kernel(KvCache c, int max_path,
                                                      const int32_t* __restrict__ seqs,
                                                      const int32_t* __restrict__ path,
                                                      const int32_t* __restrict__ n_accept) {
  __shared__ int from_s[kMaxNodes], to_s[kMaxNodes], from_p[kMaxNodes], to_p[kMaxNodes];
  const int i = blockIdx.y, acc = n_accept[i];
  if (check_commit(c, i, max_path, seqs, path, acc)) return;
  const int s = seqs[i], len = c.length[s];
  const int32_t* row = c.table + (int64_t)s * c.max_pages;
  int moved = 0;
  for (int j = threadIdx.x; j < acc; j += blockDim.x) {
    const int p = path[(int64_t)i * max_path + j];
    const int a = len + p, b = len + j;
    from_s[j] = a & (c.P - 1);
    to_s[j] = b & (c.P - 1);
    from_p[j] = row[a >> c.log_p];
    to_p[j] = row[b >> c.log_p];
    moved += p == j;
  }
  // path[j] == j for the first j0 nodes: they stay.
  const int j0 = __syncthreads_count(moved);
  if (j0 == acc) return;
  const int kp = c.D * (int)sizeof(E) / 16;        // pieces of a key
  const int units = c.L * c.Hkv * (c.D + kp);
  const int u = blockIdx.x * blockDim.x + threadIdx.x;
  if (u >= units) return;
  const int nv = c.L * c.Hkv * c.D;
  const bool is_v = u < nv;
  const int lh = is_v ? u / c.D : (u - nv) / kp, x = is_v ? u % c.D : (u - nv) % kp;
  const int64_t base = (lh / c.Hkv) * c.layer_bytes() + (lh % c.Hkv) * c.head_bytes();
  for (int j = j0; j < acc; ++j) {
    const int64_t a = base + from_p[j] * c.page_bytes(), b = base + to_p[j] * c.page_bytes();
    if (is_v) {
      const int sa = from_s[j], sb = to_s[j];
      const E* pa = reinterpret_cast<const E*>(c.v + a) + (sa >> 3) * c.D * 8 + x * 8 + (sa & 7);
      E* pb = reinterpret_cast<E*>(c.v + b) + (sb >> 3) * c.D * 8 + x * 8 + (sb & 7);
      *pb = *pa;
    } else {
      const int64_t r = (int64_t)c.D * sizeof(E);
      *reinterpret_cast<u32x4*>(c.k + b + to_s[j] * r + 16 * x) =
          *reinterpret_cast<const u32x4*>(c.k + a + from_s[j] * r + 16 * x);
    }
  }
}

__global__ __launch_bounds__(256) void kv_commit_kernel(KvCache c, int max_path,
                                                        const int32_t* __restrict__ seqs,
                                                        const int32_t* __restrict__ path,
                                                        const int32_t* __restrict__ n_accept,
                                                        int32_t* __restrict__ status) {
  const int i = blockIdx.x, acc = n_accept[i];
  const int st = check_commit(c, i, max_path, seqs, path, acc);
  if (threadIdx.x == 0) status[i] = st;
  if (st) return;
  const int s = seqs[i];
  const int64_t len = (int64_t)c.length[s] + acc;
  drop_pages(c, c.table + (int64_t)s * c.max_pages, pages_of(c, len));
  if (threadIdx.x == 0) c.length[s] = (int)len;
}

// One workgroup per token.
template <typename E>
__global__ __launch_bounds__(256) void kv_append_kernel(KvCache c, AppendArgs a) {
  const int t = blockIdx.x;
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.tok_off[mid] <= t) lo = mid; else hi = mid;
  }
  if (t < a.tok_off[lo] || t >= a.tok_off[lo + 1]) return;
  const int s = a.seqs[lo];
  if (!in_range(s, c.max_seqs)) return;
  const int64_t pos = (int64_t)c.length[s] + t - a.tok_off[lo];
  const int64_t at = pos >> c.log_p;
  if (pos < 0 || at >= c.max_pages) return;
  const int page = c.table[(int64_t)s * c.max_pages + at];
  if (!in_range(page, c.n_pages) || c.refs[page] != 1) return;
  const int slot = (int)(pos & (c.P - 1));
  const int64_t base = a.layer * c.layer_bytes() + page * c.page_bytes();
  const E* k = reinterpret_cast<const E*>(a.k) + t * a.ldk;
  const E* v = reinterpret_cast<const E*>(a.v) + t * a.ldv;
  for (int x = threadIdx.x; x < c.Hkv * c.D; x += blockDim.x) {
    const int h = x / c.D, d = x % c.D;
    const int64_t head = base + h * c.head_bytes();
    reinterpret_cast<E*>(c.k + head)[slot * c.D + d] = k[x];
    reinterpret_cast<E*>(c.v + head)[(slot >> 3) * c.D * 8 + d * 8 + (slot & 7)] = v[x];
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
  kv_reserve_kernel<<<1, 1024, 0, s>>>(c, n, seqs, extra, copied, status);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  kv_copy_kernel<<<dim3(c.L * c.Hkv, n), 256, 0, s>>>(c, seqs, copied);
  return hipGetLastError();
}

hipError_t launch_kv_commit(const KvCache& c, int n, int max_path, const int32_t* seqs,
                            const int32_t* path, const int32_t* n_accept, int32_t* status,
                            hipStream_t s) {
  if (path != nullptr && max_path > 0) {
    const int units = c.L * c.Hkv * (c.D + c.D * c.elt() / 16);
    const dim3 grid((units + 255) / 256, n);
    if (c.f32)
      kv_move_kernel<uint32_t><<<grid, 256, 0, s>>>(c, max_path, seqs, path, n_accept);
    else
      kv_move_kernel<uint16_t><<<grid, 256, 0, s>>>(c, max_path, seqs, path, n_accept);
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
  if (c.f32)
    kv_append_kernel<uint32_t><<<a.n_tokens, 256, 0, s>>>(c, a);
  else
    kv_append_kernel<uint16_t><<<a.n_tokens, 256, 0, s>>>(c, a);
  return hipGetLastError();
}

}  // namespace s2moe
