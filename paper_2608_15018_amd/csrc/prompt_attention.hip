// Causal attention of packed prompts.
//
// Rows.  As over the cache: the G = Hq / Hkv query heads of a kv head read the same
// keys, so a prompt of len tokens is len G rows, row r token r / G, and a workgroup
// takes consecutive ones.  Consecutive rows are few tokens, so little of the
// triangle's edge is computed in vain.
//
// Products (bf16).  S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 matrix
// instructions: a lane holds scores of one row, and they are, in the registers where
// the first product leaves them, the operand of the second.  Keys and values come
// through LDS, 64 tokens a stage, by loads that need no register; values, which the
// second product wants by columns, are read with LDS's transposing load.
//
// Softmax.  One pass, the running maximum moved only when it is 2^8 behind.  In bf16
// the weights enter the second product rounded to bf16 (its operands have one type);
// their sum is taken in fp32 before that.
//
// Bound: the matrix cores at D = 128 (12289 tokens, 32/4 heads: 1.16-1.22 ms, 1.02-1.06
// PFLOP/s where a large library product reaches 1.25), the weights' vector
// instructions at D = 64 (8192 tokens, 64/8 heads: 0.57-0.60 ms, 0.92-0.97 PFLOP/s);
// short prompts by what a workgroup waits for before its first product and by the
// vector instructions (24 of 512 tokens, 32/8 heads of 128: 93 us, 0.55 PFLOP/s; 24 of
// up to 1024, 64/8 heads of 64: of all cycles vector units 53 %, matrix cores 22 %, and
// 38 % of the waves' time is spent waiting).
#include "attention.h"
#include "attn_common.h"

namespace s2moe {
namespace {

// Prompts of at most so many tokens on average take 32 rows a wave, so that two or
// three workgroups share a compute unit and hide each other's starts.  us at 32 / 64
// rows a wave, 32/8 heads of 128: 96 x 128 tokens 67 / 90, 24 x 512 93 / 114, 12 x 1024
// 140 / 160, 8 x 2048 340 / 322; 64/8 heads of 64: 59 / 63, 96 / 99, 149 / 151, 357 /
// 340.  Between 1280 and 1792 tokens 128 gains and 64 loses up to 5 %.
constexpr int kShortPrompt = 1024;

// Workgroup b of a kv head: which rows of which prompt.  Prompts take
// ceil(len G / rows) workgroups each, last ones first (they see the most
// keys); 256 threads share the offsets.  None where the offsets do not ascend: prompts
// that overlap could be more workgroups than 32 bits count.
__device__ bool find_block(const PromptArgs& a, int b, int rows, int* first, int* len, int* qb) {
  __shared__ int wave_s[4], found_s[3];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = (a.n + 255) >> 8;  // consecutive prompts a thread looks at
  int n[4], f[4], mine = 0;
  bool falls = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = per * tid + i;
    n[i] = f[i] = 0;
    if (i < per && s < a.n) {
      f[i] = a.tok_off[s];
      const int end = a.tok_off[s + 1];
      falls |= end < f[i];
      n[i] = f[i] >= 0 && f[i] < end && end <= a.n_tokens ? end - f[i] : 0;
    }
    mine += (n[i] * a.G + rows - 1) / rows;
  }
  int inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  const bool any = __any(falls);
  if (lane == 63) wave_s[w] = any ? -1 : inc;
  __syncthreads();
  int at = inc - mine, total = 0, sign = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at += i < w ? wave_s[i] : 0;
    total += wave_s[i];
    sign |= wave_s[i];
  }
  if (sign < 0 || b >= total) return false;
  b = total - 1 - b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int blocks = (n[i] * a.G + rows - 1) / rows;
    if (b >= at && b < at + blocks) {
      found_s[0] = f[i];
      found_s[1] = n[i];
      found_s[2] = b - at;
    }
    at += blocks;
  }
  __syncthreads();
  *first = __builtin_amdgcn_readfirstlane(found_s[0]);
  *len = __builtin_amdgcn_readfirstlane(found_s[1]);
  *qb = __builtin_amdgcn_readfirstlane(found_s[2]);
  return true;
}

// ---------------------------------------------------------------- bf16
// NT tiles of 32 rows a wave.
template <int D, int NT>
struct PromptTile {
  static constexpr int kRows = 128 * NT;        // of a workgroup
  static constexpr int kStage = 64 * D * 2;     // bytes of 64 keys, or of their values
  static constexpr int kLoads = D / 32;         // 1 KB loads a wave makes for it
  static constexpr int kRing = NT == 2 ? 4 : 2; // stages of each in LDS
  static constexpr int kLds = 2 * kRing * kStage;
  // The overlapped loop needs all registers.
  static constexpr bool kOverlap = D == 128 && NT == 2;
  static constexpr int kPerCu = kOverlap ? 1 : D == 64 && NT == 1 ? 3 : 2;
};

template <int D, int NT>
__global__ __launch_bounds__(256, (PromptTile<D, NT>::kPerCu)) void prompt_bf16_kernel(PromptArgs a) {
  typedef PromptTile<D, NT> Tile;
  constexpr int kStage = Tile::kStage, kLoads = Tile::kLoads, kRing = Tile::kRing, kRows = Tile::kRows;
  constexpr int KS = D / 16, MT = D / 32, CH = D / 8;  // k steps, tiles of D, 16-byte chunks of a row
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* const k_lds = smem;
  char* const v_lds = smem + kRing * kStage;

  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int hk = blockIdx.x % a.Hkv;
  int first, len, qb;
  if (!find_block(a, blockIdx.x / a.Hkv, kRows, &first, &len, &qb))
    return;
  const int R = len * a.G, row0 = qb * kRows + w * 32 * NT;
  const int l32 = lane & 31, h = lane >> 5;
  const int last_row = min(qb * kRows + kRows, R) - 1;
  const int n_stage = (last_row / a.G) / 64 + 1;

  // This wave's rows: 32 steps of keys [0, n_full) that all of them see, and
  // up to n_all that some do.
  int n_full = 0, n_all = 0;
  if (row0 < R) {
    n_full = (row0 / a.G + 1) / 32;
    n_all = (min(row0 + 32 * NT - 1, R - 1) / a.G) / 32 + 1;
  }
  int tok[NT];
  const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q);
  bf16x8 qf[KS][NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = min(row0 + 32 * nt + l32, R - 1);
    tok[nt] = r / a.G;
    const uint16_t* p = q + (int64_t)(first + tok[nt]) * a.ldq + (hk * a.G + r - tok[nt] * a.G) * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks][nt] = *reinterpret_cast<const bf16x8*>(p + 16 * ks);
  }

  // Staging: chunk c of row r of a stage lies at chunk c ^ swizzle(r), so that
  // the reads below spread over all banks.  A lane's place in a stage is the
  // same for all stages; only in the last are rows past the prompt its last.
  const char* const kg = a.k + ((int64_t)first * a.ldk + hk * D) * 2;
  const char* const vg = a.v + ((int64_t)first * a.ldv + hk * D) * 2;
  const uint32_t ldk = (uint32_t)a.ldk * 2, ldv = (uint32_t)a.ldv * 2;
  const auto place = [&](int i, uint32_t ld, bool keys, int rows) {
    const int r = (w * kLoads + i) * (64 / CH) + lane / CH;
    const int x = keys ? (D == 128 ? r & 15 : (r >> 1) & 7) : (D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2);
    return (uint32_t)min(r, rows - 1) * ld + (((lane % CH) ^ x) << 4);
  };
  uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    k_off[i] = place(i, ldk, true, 64);
    v_off[i] = place(i, ldv, false, 64);
  }
  const auto load_stage = [&](const char* g, uint32_t ld, const uint32_t(&off)[kLoads], char* lds, int s, bool keys) {
    s = min(s, (len - 1) >> 6);  // past the end: the last stage again, unused
    const char* from = g + (uint64_t)s * 64 * ld;
    const int rows = len - 64 * s;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      load_to_lds(from, rows >= 64 ? off[i] : place(i, ld, keys, rows), lds + (w * kLoads + i) * 1024);
  };
  const auto load_k = [&](int s) { load_stage(kg, ldk, k_off, k_lds + (s & (kRing - 1)) * kStage, s, true); };
  const auto load_v = [&](int s) { load_stage(vg, ldv, v_off, v_lds + (s & (kRing - 1)) * kStage, s, false); };
  // Stage s is there for everybody (with four in the ring, that of the keys after it
  // too), and what is loaded now overwrites stages that nobody reads any more.
  const auto sync = [&](int s) {
    wait_loads<kRing == 4 ? 2 * kLoads : 0>();
    __builtin_amdgcn_s_barrier();
    load_k(s + kRing - 1);
    load_v(s + kRing / 2);
  };

  // Row m of a key tile is key m with bits 2 and 3 exchanged: then a lane's
  // scores 8 s .. 8 s + 7 belong to keys 16 s + 8 h + 0 .. 7, the order in
  // which the second product takes them.
  const int key_row = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
  const int k_at = key_row * D * 2, k_x = ((D == 128 ? key_row & 15 : (key_row >> 1) & 7) ^ h) << 4;
  const int v_r = (lane & 15) >> 2;
  const int v_at = (8 * h + v_r) * D * 2 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

  f32x16 O[MT][NT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) O[mt][nt] = f32x16{};
  float shift[NT], limit[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    shift[nt] = l[nt] = 0.f;
    limit[nt] = -INFINITY;
  }
  const float c = a.scale * 1.44269504088896340736f;

  const auto key_tile = [&](int j, int ks) {
    return *reinterpret_cast<const bf16x8*>(k_lds + ((j >> 1) & (kRing - 1)) * kStage + (j & 1) * 32 * D * 2 + k_at +
                                            (k_x ^ (ks << 5)));
  };
  const auto products_k = [&](int j, f32x16(&T)[NT]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) T[nt] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 kf = key_tile(j, ks);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) T[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks][nt], T[nt], 0, 0, 0);
    }
  };
  const auto value_tile = [&](int j, int ks, int mt) -> bf16x8 {
    const char* vt = v_lds + ((j >> 1) & (kRing - 1)) * kStage + ((j & 1) * 32 + 16 * ks) * D * 2 + v_at +
                     ((mt ^ (D == 128 ? v_r : v_r >> 1)) << 6);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)vt);
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(vt + 4 * D * 2));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto products_v = [&](int j, const bf16x8(&W)[2][NT]) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const bf16x8 vf = value_tile(j, ks, mt);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) O[mt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, W[ks][nt], O[mt][nt], 0, 0, 0);
      }
  };
  // The weights of one step, by the maximum as it stands.
  const auto weights = [&](const f32x16(&T)[NT], bf16x8(&W)[2][NT]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = exp2_fast(fmaf(T[nt][i], c, -shift[nt]));
        l[nt] += p[i];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) W[ks][nt] = pack8(p + 8 * ks);
    }
  };
  const auto largest = [&](const f32x16& T) {
    float m = max3(T[0], T[1], T[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) m = max3(m, T[i], T[i + 1]);
    return fmaxf(m, T[15]) * c;
  };
  // Scores of the next step whose largest are m: a row with one past its limit
  // moves its maximum there, and what it has summed so far, W's step included,
  // shrinks by 2^-8 or more (so rounding W once more does not count).
  const auto raise_to = [&](const float(&m)[NT], bf16x8(&W)[2][NT]) {
    bool over = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) over |= m[nt] > limit[nt];
    if (__builtin_expect(__any(over), 0)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float top = max_halves(m[nt]);
        const bool moves = top > limit[nt], fresh = limit[nt] == -INFINITY;
        const float f = moves && !fresh ? exp2_fast(shift[nt] - top) : 1.f;
        shift[nt] = moves ? top : shift[nt];
        limit[nt] = moves ? top + kLag : limit[nt];
        l[nt] *= f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          O[mt][nt] *= f;
          if (Tile::kOverlap) asm volatile("" : "+a"(O[mt][nt]));
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          float p[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = (float)W[ks][nt][i] * f;
          W[ks][nt] = pack8(p);
        }
      }
    }
  };
  const auto raise = [&](const f32x16(&T)[NT], bf16x8(&W)[2][NT]) {
    float m[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) m[nt] = largest(T[nt]);
    raise_to(m, W);
  };
  const auto mask = [&](int j, f32x16(&T)[NT]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * j + 16 * (i >> 3) + 8 * h + (i & 7) > tok[nt]) T[nt][i] = -INFINITY;
  };
  // The second product of step j.  Where some rows do not see some keys a weight of
  // zero does not hide an infinity or NaN, so those values count as zero there, and
  // rows that see them get what they add up to.
  const auto products_v_checked = [&](int j, bool masked, const bf16x8(&W)[2][NT]) {
    bf16x8 vf[2][MT];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) vf[ks][mt] = value_tile(j, ks, mt);
    if (masked) {
      uint32_t bad = 0;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) bad |= any_nonfinite(vf[ks][mt]);
      if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            __builtin_amdgcn_sched_barrier(0);  // one after the other: registers
            f32x16 met = {};
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
              const int n = tok[nt] + 1 - (32 * j + 16 * ks + 8 * h);  // of the eight keys
              const bf16x8 sees = sight(n < 0 ? 0 : (1u << min(n, 8)) - 1, W[ks][nt]);
              met = __builtin_amdgcn_mfma_f32_32x32x16_bf16(special_numbers(vf[ks][mt]), sees, met, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) O[mt][nt][i] += special_sum(met[i]);
          }
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) vf[ks][mt] = finite_only(vf[ks][mt]);
        }
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          O[mt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][mt], W[ks][nt], O[mt][nt], 0, 0, 0);
  };
  load_k(0);
  if constexpr (kRing == 4) load_k(1);
  load_v(0);
  if constexpr (kRing == 4) {
    load_k(2);
    load_v(1);
  }
  f32x16 SA[NT];
  bf16x8 PA[2][NT] = {};
  int s = 0;
  if constexpr (Tile::kOverlap) {
  // One step of the overlapped loop: the scores of step j + 1 into `next`, the
  // weights of step j from `now` into W, and the products of the weights
  // `before` with the values of step j - 1.  Sixteen fragments of keys and
  // values, read four ahead, with two matrix instructions each; between those,
  // two scores become weights, and then the new scores' maximum is taken.
  const auto step = [&](int j, const f32x16(&now)[NT], f32x16(&next)[NT], const bf16x8(&before)[2][NT],
                        bf16x8(&W)[2][NT], bf16x8(&ahead)[4]) {
    constexpr int NF = KS + 2 * MT, EL = 32 / NF;  // fragments, scores each
    bf16x8 f[NF + 4];
    bf16x2 w2[16];
    float m[NT];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = ahead[i];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int n = i + 4;
      if (n < KS) f[n] = key_tile(j + 1, n);
      else if (n < NF) f[n] = value_tile(j - 1, (n - KS) / MT, (n - KS) % MT);
      else f[n] = key_tile(j + 2, n - NF);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (i < KS) {
          next[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i], qf[i < KS ? i : 0][nt], i == 0 ? f32x16{} : next[nt], 0, 0, 0);
        } else {
          constexpr int dummy = 0;
          const int ks = i < KS ? dummy : (i - KS) / MT, mt = i < KS ? dummy : (i - KS) % MT;
          O[mt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i], before[ks][nt], O[mt][nt], 0, 0, 0);
        }
      }
#pragma unroll
      for (int e = i * EL; e < i * EL + EL; e += 2) {
        const int nt = e >> 4, x = e & 15;
        const float p = exp2_fast(fmaf(now[nt][x], c, -shift[nt]));
        const float r = exp2_fast(fmaf(now[nt][x + 1], c, -shift[nt]));
        l[nt] += p;
        l[nt] += r;
        w2[e >> 1] = pack2(p, r);
      }
      if (i >= KS + 2) {  // sixteen maxima over the last fragments
        constexpr int per = (16 + NF - KS - 3) / (NF - KS - 2);
#pragma unroll
        for (int g = (i - KS - 2) * per; g < (i - KS - 1) * per && g < 16; ++g) {
          const int nt = g >> 3, x = 2 * (g & 7);
          m[nt] = x == 0 ? fmaxf(next[nt][0], next[nt][1]) : max3(m[nt], next[nt][x], next[nt][x + 1]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          W[ks][nt][2 * x] = w2[8 * nt + 4 * ks + x][0];
          W[ks][nt][2 * x + 1] = w2[8 * nt + 4 * ks + x][1];
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = f[NF + i];
    asm volatile("" : "+v"(next[0]), "+v"(next[1]));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+a"(O[mt][0]), "+a"(O[mt][1]));
    m[0] *= c;
    m[1] *= c;
    raise_to(m, W);
  };
  if (n_full >= 4) {
    // Steps whose keys every row of the wave sees, two a stage, as far as they
    // are even in number.  What a step does depends on nothing else in it, so
    // the matrix cores work while the weights are made.  (At D = 64 two waves
    // share a SIMD and do this for each other.)
    f32x16 SB[NT];
    bf16x8 PB[2][NT], ahead[4];
    const int n_fast = n_full >> 1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qf[ks][0]), "+a"(qf[ks][1]));
    sync(0);
    products_k(0, SA);
    raise(SA, PA);
    products_k(1, SB);
    weights(SA, PA);
    raise(SB, PA);
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = key_tile(2, i);
    // Nothing waits for LDS before the barrier: the reads of what is loaded over
    // afterwards went into scores and sums that the step before it has used.
    for (s = 1; s < n_fast; ++s) {
      step(2 * s - 1, SB, SA, PA, PB, ahead);
      sync(s);
      step(2 * s, SA, SB, PB, PA, ahead);
    }
    weights(SB, PB);
    products_v(2 * s - 2, PA);
    products_v(2 * s - 1, PB);
  }
  }
  for (; s < n_stage; ++s) {
    wait_lds();
    sync(s);
    for (int j = 2 * s; j < 2 * s + 2 && j < n_all; ++j) {
      products_k(j, SA);
      if (j >= n_full) mask(j, SA);
      raise(SA, PA);
      weights(SA, PA);
      products_v_checked(j, j >= n_full, PA);
    }
  }
  wait_loads<0>();  // no load into this workgroup's LDS outlives it

  uint16_t* out = reinterpret_cast<uint16_t*>(a.out);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row0 + 32 * nt + l32;
    const float sum = sum_halves(l[nt]);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // 0: every score is minus infinity
    // A lane has four elements of every eight; the half-waves exchange fours, so
    // that each stores 16 bytes.
    uint16_t* p = out + (int64_t)(first + tok[nt]) * a.ldo + (hk * a.G + r - tok[nt] * a.G) * D + 8 * h;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        u32x4 v;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const bf16x2 lo = pack2(O[mt][nt][4 * b + 2 * x] * inv, O[mt][nt][4 * b + 2 * x + 1] * inv);
          const bf16x2 hi = pack2(O[mt][nt][4 * b + 4 + 2 * x] * inv, O[mt][nt][4 * b + 5 + 2 * x] * inv);
          const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, lo),
                                                             __builtin_bit_cast(uint32_t, hi), false, false);
          v[x] = both[0];
          v[2 + x] = both[1];
        }
        if (r < R) *reinterpret_cast<u32x4*>(p + 32 * mt + 8 * b) = v;
      }
  }
}

// ---------------------------------------------------------------- fp32
// The fp32 matrix instructions run at a sixteenth of the bf16 rate, so nothing needs
// LDS: a wave takes 32 rows and reads keys and values of 16 tokens a step into
// registers, the next step's as soon as this one's are used.  Their operands hold one
// k a lane, so values need no transposition: step e of a product takes key 4 g + e of
// lane group g, where the scores of those keys are.  4 prompts of 1024 tokens: 0.44 ms
// with 32/8 heads of 128 (78 TFLOP/s; a large library product reaches 153).
// SPLIT: the four waves share 32 rows and take every fourth step, and their sums
// are added at the end.
template <int D, bool SPLIT>
__global__ __launch_bounds__(256, 2) void prompt_f32_kernel(PromptArgs a) {
  constexpr int kRows = SPLIT ? 32 : 128, KC = D / 16, MT = D / 16;
  const int lane = threadIdx.x & 63, w = wave_id(), n16 = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.Hkv;
  int first, len, qb;
  if (!find_block(a, blockIdx.x / a.Hkv, kRows, &first, &len, &qb)) return;
  const int R = len * a.G, row0 = qb * kRows + (SPLIT ? 0 : w * 32);
  if (row0 >= R) return;
  const int t0 = SPLIT ? w : 0, dt = SPLIT ? 4 : 1;
  const int n_step = (min(row0 + 31, R - 1) / a.G) / 16 + 1, first_tok = row0 / a.G;

  int tok[2];
  f32x4 q[KC][2], O[MT][2];
  float shift[2] = {0.f, 0.f}, limit[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int nt = 0; nt < 2; ++nt) {
    const int row = min(row0 + 16 * nt + n16, R - 1);
    tok[nt] = row / a.G;
    const float* p = reinterpret_cast<const float*>(a.q) + (int64_t)(first + tok[nt]) * a.ldq +
                     (hk * a.G + row - tok[nt] * a.G) * D + 4 * g;
#pragma unroll
    for (int x = 0; x < KC; ++x) q[x][nt] = *reinterpret_cast<const f32x4*>(p + 16 * x);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) O[mt][nt] = f32x4{};
  }
  const float* const kg = reinterpret_cast<const float*>(a.k) + (int64_t)first * a.ldk + hk * D + 4 * g;
  const float* const vg = reinterpret_cast<const float*>(a.v) + (int64_t)first * a.ldv + hk * D + n16;
  f32x4 K[KC], V[MT];
  const auto load_k = [&](int t) {
    const float* p = kg + (int64_t)min(16 * t + n16, len - 1) * a.ldk;
#pragma unroll
    for (int x = 0; x < KC; ++x) K[x] = *reinterpret_cast<const f32x4*>(p + 16 * x);
  };
  const auto load_v = [&](int t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* p = vg + (int64_t)min(16 * t + 4 * g + e, len - 1) * a.ldv;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) V[mt][e] = p[16 * mt];
    }
  };
  const auto mma = [](f32x4 x, f32x4 y, f32x4 z) {
#pragma unroll
    for (int j = 0; j < 4; ++j) z = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], z, 0, 0, 0);
    return z;
  };
  const float c = a.scale * 1.44269504088896340736f;
  load_k(t0);
  load_v(t0);
  for (int t = t0; t < n_step; t += dt) {
    f32x4 S[2] = {};
#pragma unroll
    for (int x = 0; x < KC; ++x)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) S[nt] = mma(K[x], q[x][nt], S[nt]);
    if (t + dt < n_step) load_k(t + dt);
    const bool masked = 16 * t + 15 > first_tok;
    float m[2];
    bool over = false;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      if (masked)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * t + 4 * g + e > tok[nt]) S[nt][e] = -INFINITY;
      m[nt] = fmaxf(max3(S[nt][0], S[nt][1], S[nt][2]), S[nt][3]) * c;
      over |= m[nt] > limit[nt];
    }
    if (__any(over)) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
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
    f32x4 P[2];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        P[nt][e] = exp2_fast(fmaf(S[nt][e], c, -shift[nt]));
        l[nt] += P[nt][e];
      }
    if (masked) {  // as in the bf16 kernel
      uint32_t bad = 0;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) bad |= any_nonfinite(V[mt]);
      if (__any(bad != 0))
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            __builtin_amdgcn_sched_barrier(0);  // one after the other: registers
            const int n = tok[nt] + 1 - (16 * t + 4 * g);  // of the four keys
            const f32x4 met = mma(special_numbers(V[mt]), sight(n < 0 ? 0 : (1u << min(n, 4)) - 1, P[nt]), f32x4{});
#pragma unroll
            for (int e = 0; e < 4; ++e) O[mt][nt][e] += special_sum(met[e]);
          }
          V[mt] = finite_only(V[mt]);
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) O[mt][nt] = mma(V[mt], P[nt], O[mt][nt]);
    if (t + dt < n_step) load_v(t + dt);
  }
  if constexpr (SPLIT) {
    __shared__ __attribute__((aligned(16))) float o_s[3][2][MT][64][4];
    __shared__ float m_s[4][2][16], l_s[4][2][16];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      l[nt] = sum_groups(l[nt]);
      m_s[w][nt][n16] = limit[nt] == -INFINITY ? -INFINITY : shift[nt];
      l_s[w][nt][n16] = l[nt];
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) top = fmaxf(top, m_s[x][nt][n16]);
#pragma unroll
      for (int x = 0; x < 4; ++x)
        sum += l_s[x][nt][n16] * (m_s[x][nt][n16] == -INFINITY ? 0.f : exp2_fast(m_s[x][nt][n16] - top));
      const float own = m_s[w][nt][n16], f = own == -INFINITY ? 0.f : exp2_fast(own - top);
      l[nt] = sum;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        O[mt][nt] *= f;
        if (w > 0) *reinterpret_cast<f32x4*>(o_s[w - 1][nt][mt][lane]) = O[mt][nt];
      }
    }
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int x = 0; x < 3; ++x)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) O[mt][nt] += *reinterpret_cast<const f32x4*>(o_s[x][nt][mt][lane]);
  }
#pragma unroll
  for (int nt = 0; nt < 2; ++nt) {
    const int row = row0 + 16 * nt + n16;
    const float sum = SPLIT ? l[nt] : sum_groups(l[nt]);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // as in the bf16 kernel
    if (row >= R) continue;
    float* p = reinterpret_cast<float*>(a.out) + (int64_t)(first + tok[nt]) * a.ldo +
               (hk * a.G + row - tok[nt] * a.G) * D + 4 * g;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4*>(p + 16 * mt) = O[mt][nt] * inv;
  }
}

template <int D, int NT>
hipError_t launch_bf16(const PromptArgs& a, hipStream_t s) {
  typedef PromptTile<D, NT> Tile;
  static std::atomic<uint64_t> ready{0};
  const hipError_t err = allow_lds(reinterpret_cast<const void*>(prompt_bf16_kernel<D, NT>), Tile::kLds, ready);
  if (err != hipSuccess) return err;
  // At most one unfilled workgroup per prompt.
  const int64_t blocks = ((int64_t)a.n_tokens * a.G / Tile::kRows + a.n) * a.Hkv;
  prompt_bf16_kernel<D, NT><<<(unsigned)blocks, 256, Tile::kLds, s>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_bf16(const PromptArgs& a, hipStream_t s) {
  // Also where 64 rows a wave would make hardly more than the workgroups that run at
  // once.  us at 32 / 64 rows a wave, one prompt, 32/8 heads of 128: 1536 tokens 42 / 50,
  // 2048 57 / 63, 4000 148 / 137; 64/8 heads of 64: 33 / 44, 48 / 57, 3000 98 / 91.
  typedef PromptTile<D, 2> Wide;
  const int64_t wide = ((int64_t)a.n_tokens * a.G / Wide::kRows + a.n) * a.Hkv;
  const bool few = wide <= 288 * Wide::kPerCu;
  return few || a.n_tokens / a.n <= kShortPrompt ? launch_bf16<D, 1>(a, s) : launch_bf16<D, 2>(a, s);
}

template <int D>
hipError_t launch_f32(const PromptArgs& a, hipStream_t s) {
  // By keys while rows alone would not give every SIMD of the GPU a wave, and for long
  // prompts, whose workgroups of 32 rows end more evenly than those of 128.  us by keys
  // / by rows: 3 x 150 tokens, 4/2 heads of 64, 9 / 16; 8 x 2000 201 / 319; 32/8 heads of
  // 128: 64 x 64 99 / 59, 32 x 128 121 / 103, 16 x 256 167 / 188, 4 x 1024 443 / 567,
  // 1 x 4096 1511 / 1721 (but 4 x 256 54 / 45); of 64: 32 x 128 70 / 57, 4 x 1024 215 / 292.
  const auto blocks = [&](int rows) { return ((int64_t)a.n_tokens * a.G / rows + a.n) * a.Hkv; };
  if (blocks(32) < 1024 || a.n_tokens / a.n >= 256)
    prompt_f32_kernel<D, true><<<(unsigned)blocks(32), 256, 0, s>>>(a);
  else
    prompt_f32_kernel<D, false><<<(unsigned)blocks(128), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t s) {
  if (!a.f32) return a.D == 64 ? launch_bf16<64>(a, s) : launch_bf16<128>(a, s);
  return a.D == 64 ? launch_f32<64>(a, s) : launch_f32<128>(a, s);
}

}  // namespace s2moe
