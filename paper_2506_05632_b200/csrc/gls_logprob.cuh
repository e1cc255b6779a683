// gls_logprob.cuh -- log probabilities of given tokens with the row's entropy and its most likely
// alternatives, and their gradient with respect to the logits.
//
// Per row x of V logits, with z = x / T over the finite logits of the row (NaN, +inf and -inf are
// masked, as everywhere in the library):
//     lse = ln sum_i e^(z_i),   p_i = e^(z_i - lse),   log probability of token t = z_t - lse,
//     H = -sum_i p_i ln p_i = ln s - u / T / s  with s = sum_i e^(z_i - z_m), u = sum_i e^(z_i - z_m) (x_i - x_m)
// for any reference x_m, so one pass over the row yields all of it, and the M largest logits of
// the same pass (descending, ties to the lower index) are the alternatives.
#pragma once
#include <cstddef>
#include <type_traits>

#include "gls_group16.cuh"

namespace gls {

constexpr int kScoreMaxM = 256;          // alternatives per row
constexpr int kScoreMaxG = 64;           // given tokens per row
constexpr uint32_t kDevBadToken = 2u;    // GLS_DEV_BAD_TOKEN

struct ScoreArgs {
  const void* data;       // rows [B][K][J][V]
  long long sb, sk, sj;   // element strides
  int K, J, V, M, G;
  int emitted;            // 1: row (b, j) is that of the lowest draft active at j (see accept)
  int L;
  const uint8_t* accept;  // [B][K][L]
  long long rows;         // B * K * J, or B * J for emitted rows
  const int32_t* tokens;  // [rows][G]
  float inv_t[kMaxK];
  float* out_lp;          // [rows][G]
  float* out_lse;         // [rows]
  float* out_tail;        // NULL or [rows]: lse - out_lse in the precision that fp32 leaves
  float* out_ent;         // NULL or [rows]
  int32_t* top_ids;       // [rows][M]
  float* top_lp;          // [rows][M]
  uint32_t* status;
};

struct ScoreRow {
  const char* rowp;
  float inv_t;
  bool live;  // false: an emitted row behind the last token; it is not read
};

template <int ES>
__device__ __forceinline__ ScoreRow score_locate(const ScoreArgs& A, long long row) {
  ScoreRow r;
  const int lane = threadIdx.x & 31;
  int k;
  long long b;
  const uint32_t bk = (uint32_t)row / (uint32_t)A.J;  // rows number fewer than 2^25
  const int j = (int)((uint32_t)row - bk * (uint32_t)A.J);
  if (A.emitted) {
    b = bk;
    k = 0;
    const int t = __ldg(A.tokens + row);
    if (j > 0) {  // lowest draft whose position j - 1 was accepted; read beside the token
      const uint8_t* a = A.accept + b * A.K * A.L + (j - 1);
      const unsigned lo = __ballot_sync(0xffffffffu, lane < A.K && __ldg(a + (long long)lane * A.L) != 0);
      const unsigned hi = A.K > 32 ? __ballot_sync(0xffffffffu, lane + 32 < A.K && __ldg(a + (long long)(lane + 32) * A.L) != 0) : 0u;
      k = lo != 0u ? __ffs(lo) - 1 : hi != 0u ? 31 + __ffs(hi) : 0;
    }
    r.live = t >= 0;
  } else {
    b = bk / (uint32_t)A.K;
    k = (int)(bk - (uint32_t)b * (uint32_t)A.K);
    r.live = true;
  }
  r.inv_t = A.inv_t[k];
  r.rowp = (const char*)A.data + (b * A.sb + (long long)k * A.sk + (long long)j * A.sj) * ES;
  return r;
}

// A row is read in groups of 16 tokens counted from the 32-byte boundary at or below its start, so
// that a row that starts anywhere is read by aligned 32-byte loads.  `mis`: elements between that
// boundary and the row's start; `end`: mis + V.  Virtual index v is token v - mis.
template <int DT>
struct ScoreCfg {  // one step of a warp: 4 KB of the row
  static constexpr int kGroups = DT == kBF16 ? 4 : 2;  // groups of 16 tokens per lane
  static constexpr int kStep = 512 * kGroups;
};

// A group that sticks out of the row at either end, element by element.  What is outside becomes
// the lowest finite value: its exponential is exactly 0 and its product with a difference too.
template <int DT>
__device__ __noinline__ void score_edge(Group16<DT>* g, const char* rowp, int v, int mis, int end) {
  if constexpr (DT == kBF16) {
#pragma unroll 1
    for (int t = 0; t < 8; ++t) {
      const int a = v + 2 * t;
      const uint32_t lo = a >= mis && a < end ? (uint32_t)__ldg((const unsigned short*)rowp + (a - mis)) : 0xff7fu;
      const uint32_t hi = a + 1 >= mis && a + 1 < end ? (uint32_t)__ldg((const unsigned short*)rowp + (a + 1 - mis)) : 0xff7fu;
      g->a.w[t] = lo | (hi << 16);
    }
  } else {
    uint32_t* const w = (uint32_t*)g;
#pragma unroll 1
    for (int t = 0; t < 16; ++t) {
      const int a = v + t;
      w[t] = a >= mis && a < end ? __float_as_uint(__ldg((const float*)rowp + (a - mis))) : 0xff7fffffu;
    }
  }
}
template <int DT>
__device__ __forceinline__ void score_load(Group16<DT> (&g)[ScoreCfg<DT>::kGroups], const char* rowp, int mis, int end,
                                           int step) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int kStep = ScoreCfg<DT>::kStep;
  const int s0 = step * kStep;
  const int v0 = s0 + (threadIdx.x & 31) * 16;
  const char* const p = rowp + ((long long)v0 - mis) * ES;
  if (s0 >= mis && s0 + kStep <= end) {
#pragma unroll
    for (int q = 0; q < ScoreCfg<DT>::kGroups; ++q) load16_vec(g[q], p + q * 512 * ES);
  } else {
#pragma unroll
    for (int q = 0; q < ScoreCfg<DT>::kGroups; ++q) {
      const int v = v0 + q * 512;
      if (v >= mis && v + 16 <= end) {
        load16_vec(g[q], p + q * 512 * ES);
      } else {
        Group16<DT> e;
        score_edge<DT>(&e, rowp, v, mis, end);
        g[q] = e;
      }
    }
  }
}

// Softmax statistics relative to the reference logit m; s == 0: no finite logit.
struct ScoreSums {
  float m, s, u;
};

// Adds one step of a lane's groups to its sums.  The reference moves only when the step's maximum
// mx exceeds it by 2^8, so that terms stay within fp32 and the two parts of the entropy small.  A
// step's terms are added up by themselves first: a lane's chain of additions is 32 + V / (32 step)
// long.  The difference to the reference is taken before the scale: it is exact, or rounded at
// 2^-24 of itself, so an exponent is good to 1e-7 of its own size however large the logits are.
// -inf and NaN make the step's sums NaN (a masked vocabulary tail is common, a masked step in the
// middle is not); such a step is taken again with both set to the lowest finite value, whose terms
// are exactly 0, and the row's further steps are taken that way at once.  +inf makes the sums infinite, which the caller finds at the end.
template <int DT, bool ENT, bool CLAMP>
__device__ __forceinline__ void score_terms(const Group16<DT> (&g)[ScoreCfg<DT>::kGroups], float lm, float c2,
                                            float& s, float& u) {
  const unsigned long long c22 = pack_f32x2(c2, c2), nlm2 = pack_f32x2(-lm, -lm);
  constexpr int NG = ScoreCfg<DT>::kGroups;
  unsigned long long s2[NG], u2[NG];  // a chain of additions per group: they overlap
#pragma unroll
  for (int q = 0; q < NG; ++q) {
    s2[q] = u2[q] = 0ull;
    Group16<DT> h = g[q];
    if (CLAMP) {
      if constexpr (DT == kBF16) {
#pragma unroll
        for (int t = 0; t < 8; ++t) h.a.w[t] = max_bf16x2(h.a.w[t], 0xff7fff7fu);
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          h.a.w[t] = __float_as_uint(fmaxf(__uint_as_float(h.a.w[t]), -3.402823466e38f));
          h.b.w[t] = __float_as_uint(fmaxf(__uint_as_float(h.b.w[t]), -3.402823466e38f));
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 16; t += 2) {
      const unsigned long long d2 = group16_diff2(h, t, -lm, nlm2);
      float e0, e1;
      unpack_f32x2(mul_f32x2(d2, c22), e0, e1);
      const unsigned long long e2 = pack_f32x2(ex2_approx(e0), ex2_approx(e1));
      s2[q] = add_f32x2(s2[q], e2);
      if (ENT) u2[q] = fma_f32x2(e2, d2, u2[q]);
    }
  }
#pragma unroll
  for (int d = NG / 2; d > 0; d >>= 1) {
#pragma unroll
    for (int q = 0; q < d; ++q) {
      s2[q] = add_f32x2(s2[q], s2[q + d]);
      if (ENT) u2[q] = add_f32x2(u2[q], u2[q + d]);
    }
  }
  float a0, a1;
  unpack_f32x2(s2[0], a0, a1);
  s = a0 + a1;
  unpack_f32x2(u2[0], a0, a1);
  u = a0 + a1;
}
template <int DT, bool ENT>
__device__ __forceinline__ void score_step(const Group16<DT> (&g)[ScoreCfg<DT>::kGroups], float mx, float c2,
                                           ScoreSums& t, bool& masked) {
  if (fmaf(mx - t.m, c2, -8.0f) > 0.f && mx < CUDART_INF_F) {
    const float r = ex2_approx((t.m - mx) * c2);
    if (ENT) t.u = r > 0.f ? r * (t.u + t.s * (t.m - mx)) : 0.f;  // x - mx = (x - m) + (m - mx)
    t.s *= r;
    t.m = mx;
  }
  float s, u;
  if (!masked) {
    score_terms<DT, ENT, false>(g, t.m, c2, s, u);
    masked = __any_sync(0xffffffffu, ENT ? u != u : s != s);
  }
  if (masked) score_terms<DT, ENT, true>(g, t.m, c2, s, u);
  t.s += s;
  if (ENT) t.u += u;
}

// Maximum of a lane's tokens of a step, NaN ignored (NaN if there is nothing else).
template <int DT>
__device__ __forceinline__ float score_max(const Group16<DT> (&g)[ScoreCfg<DT>::kGroups]) {
  if constexpr (DT == kBF16) {
    uint32_t x = g[0].a.w[0];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < 8; ++t)
        if (q + t > 0) x = max_bf16x2(x, g[q].a.w[t]);
    return fmaxf(bf16_lo(x), bf16_hi(x));
  } else {
    return fmaxf(group16_max(g[0]), group16_max(g[1]));
  }
}

template <int DT>
__device__ __forceinline__ float score_group_max(const Group16<DT>& g) {
  if constexpr (DT == kBF16) {
    uint32_t x = g.a.w[0];
#pragma unroll
    for (int t = 1; t < 8; ++t) x = max_bf16x2(x, g.a.w[t]);
    return fmaxf(bf16_lo(x), bf16_hi(x));
  } else {
    return group16_max(g);
  }
}

// A lower bound on the k-th largest of the warp's 32 N values (ordered codes), exact in its upper
// 16 bits at least.  0 when fewer than k are above 0.  A few are taken off the top one by one (80
// cycles each); otherwise the code is found two bits at a time.
template <int N>
__device__ __forceinline__ uint32_t warp_kth(const uint32_t (&code)[N], int k) {
  uint32_t kth = 0u;
  if (k <= 6) {
    uint32_t v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = code[q];
#pragma unroll 1
    for (int i = 0; i < k; ++i) {
      uint32_t mine = v[0];
#pragma unroll
      for (int q = 1; q < N; ++q) mine = max(mine, v[q]);
      kth = __reduce_max_sync(0xffffffffu, mine);
      const unsigned who = __ballot_sync(0xffffffffu, mine == kth);
      bool drop = (int)(threadIdx.x & 31) == __ffs(who) - 1;
#pragma unroll
      for (int q = 0; q < N; ++q) {
        if (drop && v[q] == kth) {
          v[q] = 0u;
          drop = false;
        }
      }
    }
    return kth;
  }
  // the bits that all values above 0 share need no search
  uint32_t hi = code[0], lo = code[0] - 1u;
#pragma unroll
  for (int q = 1; q < N; ++q) {
    hi = max(hi, code[q]);
    lo = min(lo, code[q] - 1u);  // 0 wraps to the top
  }
  hi = __reduce_max_sync(0xffffffffu, hi);
  lo = __reduce_min_sync(0xffffffffu, lo) + 1u;
  if (hi == 0u) return 0u;
  const int free_bits = 32 - __clz(hi ^ lo);
  int shift = free_bits > 16 ? (free_bits - 1) & ~1 : 14;
  kth = shift >= 30 ? 0u : hi >> (shift + 2) << (shift + 2);
  {  // fewer than k values above 0: no bound
    uint32_t c = 0u;
#pragma unroll
    for (int q = 0; q < N; ++q) c += code[q] > 0u ? 1u : 0u;
    if (__reduce_add_sync(0xffffffffu, c) < (uint32_t)k) return 0u;
  }
#pragma unroll 1
  for (; shift >= 16; shift -= 2) {
    // how many values are at or above each of the three next thresholds: at most 512, ten bits each
    uint32_t c = 0u;
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      const uint32_t t = kth | ((uint32_t)(d + 1) << shift);
#pragma unroll
      for (int q = 0; q < N; ++q) c += code[q] >= t ? 1u << (10 * d) : 0u;
    }
    c = __reduce_add_sync(0xffffffffu, c);
    const uint32_t k_ = (uint32_t)k;
    kth |= (uint32_t)(((c & 1023u) >= k_) + (((c >> 10) & 1023u) >= k_) + ((c >> 20) >= k_)) << shift;
  }
  return kth;
}
// ------------------------------------------------------------------------------------------
// The M largest logits.  The sweep itself only stores, per lane and step, the largest of the lane's
// tokens ("entry": 64 tokens of bf16, 32 of fp32, or a power of two of steps where there would be
// too many), rounded down to bf16: two instructions a step.  At the end the M-th largest of a few
// maxima over entries (distinct tokens) bounds the M-th largest logit T from below; entries that
// reach T are listed, their tokens read once more, and those that reach T ranked.  About a tenth more
// than M tokens get that far where large logits lie anywhere in the row.  (Testing groups
// against a running threshold in the sweep and examining them in batches took 11 thousand
// instructions a row of 152064 tokens and M = 20, four tenths of what the sums take.)
// Where large logits lie side by side, the entries hide all but one of each 64 (32) of them and T is far
// below the M-th largest; in the cluster kernel, whose bound is the smallest of its warps', even more so.
// Rows of which more tokens reach T than the buffers hold, these or rows of equal logits, go through a radix
// select, which reads the whole row for each of its passes.  Rows in the order of 2 ln(rank) with noise of 1,
// beside the same shuffled: one of 152064, M = 5, 39 us and 10; 224 of 128256, M = 20, 125 and 21; 8192 of
// 152064, M = 20, 454 and 423, M = 50, 7.1 ms and 0.45, M = 256, 10.1 and 0.74.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t top_entry_bits(float x, std::integral_constant<int, kBF16>) {
  return __float_as_uint(x) >> 16;
}
// x rounded down to bf16
__device__ __forceinline__ uint32_t bf16_floor_bits(float x) {
  uint32_t b = __float_as_uint(x);
  if (b & 0x80000000u) b += 0xffffu;
  return b >> 16;
}
__device__ __forceinline__ uint32_t top_entry_bits(float x, std::integral_constant<int, kF32>) {
  return bf16_floor_bits(x);
}
// log2 of the steps per entry for at most `most` entries
__device__ __forceinline__ int entry_shift(int steps, int most) {
  int k = 0;
  while (((steps - 1) >> k) >= most) ++k;
  return k;
}
// A lane's column of entries: word w holds entries 2 w and 2 w + 1, words 32 apart.
struct EntryColumn {
  uint32_t* col;  // + lane already
  int n;          // entries
  __device__ __forceinline__ void put(int e, uint32_t bits) { ((uint16_t*)(col + (e >> 1) * 32))[e & 1] = (uint16_t)bits; }
  __device__ __forceinline__ int words() const { return (n + 1) >> 1; }
};
constexpr uint32_t kNoEntry2 = 0xff80ff80u;  // -inf twice

// Maxima of a lane's entries, eight pairs.  An entry of +inf is left out: nothing is known about its
// finite tokens.
__device__ __forceinline__ void entry_slots(const EntryColumn& c, uint32_t (&acc)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = kNoEntry2;
  const int W = c.words();
#pragma unroll 1
  for (int w0 = 0; w0 < W; w0 += 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (w0 + j < W) acc[j] = max_bf16x2(acc[j], c.col[(w0 + j) * 32]);
  }
  uint32_t any = acc[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) any = max_bf16x2(any, acc[j]);
  if ((any & 0xffffu) == 0x7f80u || (any >> 16) == 0x7f80u) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = kNoEntry2;
    for (int w = 0; w < W; ++w) {
      uint32_t x = c.col[w * 32];
      if ((x & 0xffffu) == 0x7f80u) x = (x & 0xffff0000u) | 0xff80u;
      if ((x >> 16) == 0x7f80u) x = (x & 0xffffu) | 0xff800000u;
      acc[0] = max_bf16x2(acc[0], x);
    }
  }
}
// Ordered codes of N pairs; 0 where there is no finite logit.
template <int N>
__device__ __forceinline__ uint32_t slots_kth(const uint32_t (&pair)[N], int k) {
  uint32_t code[2 * N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float lo = bf16_lo(pair[j]), hi = bf16_hi(pair[j]);
    code[2 * j] = lo > -CUDART_INF_F ? enc_ordered(lo + 0.0f) : 0u;
    code[2 * j + 1] = hi > -CUDART_INF_F ? enc_ordered(hi + 0.0f) : 0u;
  }
  return warp_kth<2 * N>(code, k);
}
// The warp's bound: at least k of its tokens have this code or more (0: no bound).  512 maxima for many
// tokens, 128 for few.
__device__ __forceinline__ uint32_t entry_bound(const EntryColumn& c, int k) {
  uint32_t acc[8];
  entry_slots(c, acc);
  if (k > 64) return slots_kth<8>(acc, k);
  const uint32_t few[2] = {max_bf16x2(max_bf16x2(acc[0], acc[2]), max_bf16x2(acc[4], acc[6])),
                           max_bf16x2(max_bf16x2(acc[1], acc[3]), max_bf16x2(acc[5], acc[7]))};
  return slots_kth<2>(few, k);
}
// What an entry and a token have to exceed to reach the bound.
struct EntryTest {
  bool all;       // no bound: every entry
  uint32_t low2;  // the bf16 below the bound, twice
  float thr;      // tokens strictly above it
};
__device__ __forceinline__ EntryTest entry_test(uint32_t bound) {
  EntryTest t;
  const uint32_t o = bound >> 16;
  t.all = o <= 0x007fu;  // at or below the code of -inf
  const uint32_t d = o - 1u;
  uint32_t raw = (d & 0x8000u) ? d & 0x7fffu : ~d & 0xffffu;
  if (raw == 0x8000u) raw = 0x8001u;  // below +0 comes the largest negative number, not -0
  t.low2 = raw * 0x10001u;
  const float f = dec_ordered(o << 16);
  t.thr = t.all ? -CUDART_INF_F : __uint_as_float(o == 0x8000u ? 0x80000001u : o > 0x8000u ? __float_as_uint(f) - 1u : __float_as_uint(f) + 1u);
  return t;
}
// Lists the entries of the warp's lanes that pass, ids e * 32 + lane + base, behind what *count says; the
// caller's warps may share the list.
template <int WORDS>
__device__ __forceinline__ void entry_list(const EntryColumn& c, const EntryTest& t, uint16_t* list, int cap, int* count,
                                           int base) {
  const int lane = threadIdx.x & 31;
  constexpr int kMasks = (WORDS + 15) / 16;
  uint32_t pass[kMasks];  // a bit per entry
  int n = 0;
#pragma unroll
  for (int j = 0; j < kMasks; ++j) {
    pass[j] = 0u;
    if (16 * j >= c.words()) continue;
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int w = j * 16 + i;
      if (w < WORDS && w < c.words()) {
        const uint32_t x = max_bf16x2(c.col[w * 32], t.low2) ^ t.low2;
        if ((x & 0xffffu) != 0u || t.all) m |= 1u << (2 * i);
        if ((x >> 16) != 0u || t.all) m |= 2u << (2 * i);
      }
    }
    const int left = c.n - 32 * j;
    if (left < 32) m &= (1u << left) - 1u;
    pass[j] = m;
    n += __popc(m);
  }
  int incl = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  int at = 0;
  if (lane == 31) at = atomicAdd(count, incl);
  at = __shfl_sync(0xffffffffu, at, 31) + incl - n;
#pragma unroll
  for (int j = 0; j < kMasks; ++j) {
    for (uint32_t m = pass[j]; m != 0u; m &= m - 1u, ++at)
      if (at < cap) list[at] = (uint16_t)(base + (32 * j + __ffs(m) - 1) * 32 + lane);
  }
}
__device__ __forceinline__ unsigned long long score_code(uint32_t key, int idx) {
  return ((unsigned long long)key << 32) | (uint32_t)~idx;  // orders by value, then by lower index
}
__device__ __forceinline__ void copy16_async(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
// Requests the group at virtual index v into shared memory (cp.async.wait_all by the same thread).
template <int DT>
__device__ __forceinline__ void group_fetch(Group16<DT>* to, const char* rowp, int v, int mis, int end) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  if (v >= mis && v + 16 <= end) {
    const char* const p = rowp + ((long long)v - mis) * ES;
#pragma unroll
    for (int h = 0; h < 16 * ES / 16; ++h) copy16_async((char*)to + 16 * h, p + 16 * h);
  } else if (v < end) {
    score_edge<DT>(to, rowp, v, mis, end);
  }
}
// Appends the tokens above thr of a group in shared memory to the candidates.
template <int DT>
__device__ __forceinline__ void group_candidates(const Group16<DT>* from, int v, int mis, int end, float thr,
                                                 unsigned long long* cand, int cap, int* count) {
  const Group16<DT> g = *from;
  uint32_t pass = 0u;
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    const float x = group16_get<DT>(g, t);
    if (x > thr && x < CUDART_INF_F) pass |= 1u << t;  // false for NaN
  }
  if (v < mis) pass &= 0xffffu << (mis - v);  // outside the row
  if (v + 16 > end) pass &= 0xffffu >> (v + 16 - end);
  if (pass == 0u) return;
  int at = atomicAdd(count, __popc(pass));
  for (; pass != 0u; pass &= pass - 1u, ++at) {
    const int t = __ffs(pass) - 1;
    const float x = DT == kF32 ? ((const float*)from)[t] : __uint_as_float((uint32_t)((const uint16_t*)from)[t] << 16);
    if (at < cap) cand[at] = score_code(enc_ordered(x + 0.0f), v + t - mis);
  }
}

// The rank of each of n candidates, by counting those before it; a thread takes every `stride`-th from
// `first`, four at a time where there are many.
template <class F>
__device__ __forceinline__ void rank_candidates(const unsigned long long* cand, int n, int first, int stride, F&& put) {
  int i = first;
  for (; i + stride < n; i += 4 * stride) {
    unsigned long long c[4];
    int r[4] = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] = i + q * stride < n ? cand[i + q * stride] : 0ull;
#pragma unroll 2
    for (int o = 0; o < n; ++o) {
      const unsigned long long x = cand[o];
#pragma unroll
      for (int q = 0; q < 4; ++q) r[q] += x > c[q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (i + q * stride < n) put(r[q], c[q]);
  }
  if (i < n) {
    const unsigned long long c = cand[i];
    int r = 0;
    for (int o = 0; o < n; ++o) r += cand[o] > c;
    put(r, c);
  }
}

// The M best tokens among the steps first, first + stride, .. of the caller's warps, and perhaps more, `cap`
// in all: a radix select over (value, index) codes, eight bits a pass from the top, each pass reading the
// steps again, until what is at or above the M-th code's bits fits; then these tokens, in no order.
// THREADS: 32 (a warp) or a whole CTA.
struct SelectShared {
  uint32_t hist[256];
  uint32_t bin, rem, count;
};
template <int DT, int THREADS>
__device__ __noinline__ void score_select(SelectShared& sh, unsigned long long* cand, int* n_cand, const char* rowp,
                                          int mis, int end, int first, int stride, int M, int cap) {
  constexpr int kStep = ScoreCfg<DT>::kStep;
  constexpr int kAhead = 8;
  const int tid = THREADS == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x, lane = threadIdx.x & 31;
  auto sync = [&]() {
    if (THREADS == 32) __syncwarp();
    else __syncthreads();
  };
  auto for_each = [&](auto&& f) {
    for (long long s = first; s * kStep < end; s += stride) {
      for (int t = lane; t < kStep; t += 32 * kAhead) {
        const long long v = s * kStep + t;
        float x[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
          x[q] = v + 32 * q >= mis && v + 32 * q < end ? load_logit<DT>(rowp, v + 32 * q - mis) : CUDART_INF_F;
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
          if (fabsf(x[q]) < CUDART_INF_F) f(score_code(enc_ordered(x[q] + 0.0f), (int)(v + 32 * q - mis)));
      }
    }
  };
  unsigned long long prefix = 0ull;
  uint32_t remaining = (uint32_t)M;
  int shift = 56;
  for (;;) {
    sync();
    for (int i = tid; i < 256; i += THREADS) sh.hist[i] = 0u;
    sync();
    for_each([&](unsigned long long c) {
      if (shift == 56 || (c >> (shift + 8)) == prefix) atomicAdd(&sh.hist[(c >> shift) & 255u], 1u);
    });
    sync();
    if (tid < 32) {  // eight bins a lane, from the top
      int bin = 255 - 8 * lane;
      uint32_t mine = 0u;
#pragma unroll
      for (int b = 0; b < 8; ++b) mine += sh.hist[bin - b];
      uint32_t incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      uint32_t above = incl - mine;
      if (above < remaining && (incl >= remaining || lane == 31)) {
        const int last = bin - 7;
        for (; bin > last && above + sh.hist[bin] < remaining; --bin) above += sh.hist[bin];
        sh.bin = (uint32_t)bin;
        sh.rem = remaining - above;  // more than the bin's count when there are fewer than M tokens
        sh.count = sh.hist[bin];
      }
    }
    sync();
    prefix = (prefix << 8) | sh.bin;
    remaining = sh.rem;
    // every code with this prefix is wanted, or can be had with those above it
    if (sh.count <= remaining || (uint32_t)M - remaining + sh.count <= (uint32_t)cap || shift == 0) break;
    shift -= 8;
  }
  const unsigned long long from = prefix << shift;
  sync();
  if (tid == 0) *n_cand = 0;
  sync();
  for_each([&](unsigned long long c) {
    if (c >= from) {
      const int at = atomicAdd(n_cand, 1);
      if (at < cap) cand[at] = c;
    }
  });
  sync();
}

// Statistics of tokens t0, t0 + dt, .. below V (each thread its own) with every element checked, two
// passes, sums in 64 bits: for rows on which the sweep's arithmetic does not hold (+inf logits,
// logits beyond 1e30 in size, no finite logit at all).  First the maximum, then the sums.
template <int DT>
__device__ __noinline__ float careful_max(const char* rowp, int t0, int dt, int V) {
  float m = -CUDART_INF_F;
  for (long long t = t0; t < V; t += dt) {
    const float x = load_logit<DT>(rowp, t);
    if (fabsf(x) < CUDART_INF_F) m = fmaxf(m, x);
  }
  return m;
}
template <int DT>
__device__ __noinline__ double2 careful_sums(const char* rowp, int t0, int dt, int V, float m, float c2) {
  double s = 0.0, u = 0.0;
  for (long long t = t0; t < V; t += dt) {
    const float x = load_logit<DT>(rowp, t);
    if (!(fabsf(x) < CUDART_INF_F)) continue;
    const double d = (double)x - (double)m;
    const double e = exp2(d * (double)c2);
    s += e;
    if (e > 0.0) u += e * d;
  }
  return make_double2(s, u);
}
__device__ __forceinline__ double2 warp_sum2(double2 a) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a.x += __shfl_xor_sync(0xffffffffu, a.x, d);
    a.y += __shfl_xor_sync(0xffffffffu, a.y, d);
  }
  return a;
}
__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  return m;
}
// Sums relative to the reference from, moved to the reference m.
__device__ __forceinline__ double2 part_at(double2 a, float from, float m, float c2) {
  const float r = ex2_approx((from - m) * c2);
  if (!(r > 0.f)) return make_double2(0.0, 0.0);
  return make_double2(a.x * (double)r, (a.y + a.x * ((double)from - (double)m)) * (double)r);
}
// The lane's sums moved to the reference m; NaN when they are not finite, however far below m.
__device__ __forceinline__ double2 sums_at(const ScoreSums& t, float m, float c2) {
  if (!(t.s < CUDART_INF_F)) return make_double2(CUDART_NAN, CUDART_NAN);
  return part_at(make_double2((double)t.s, (double)t.u), t.m, m, c2);
}
// Whether the sweep's sums stand: not zero, infinite or NaN, and the reference in the range in which
// a difference of two logits can not overflow.
__device__ __forceinline__ bool sums_stand(double2 a, float m) {
  return a.x > 0.0 && a.x < (double)CUDART_INF_F && fabs(a.y) < (double)CUDART_INF_F && m < 1e30f;
}

// The given token of this lane and its logit, requested before the row is read.
struct ScoreGiven {
  int t;
  float x;
};
template <int DT>
__device__ __forceinline__ ScoreGiven score_given(const ScoreArgs& A, long long row, const ScoreRow& rl, int g) {
  ScoreGiven r = {-1, 0.f};
  if (g < A.G) {
    r.t = __ldg(A.tokens + row * A.G + g);
    if (r.t >= 0 && r.t < A.V) r.x = load_logit<DT>(rl.rowp, r.t);
  }
  return r;
}

// Outputs of one row except its alternatives, by one warp.  m reference logit, s and u the sums, ls the
// logarithm of s (0 without a finite logit).
template <int DT>
__device__ __forceinline__ void score_emit(const ScoreArgs& A, long long row, const ScoreRow& rl, ScoreGiven gv,
                                           float m, double s, double u, double ls) {
  const int lane = threadIdx.x & 31;
  const bool some = s > 0.0;
  const double lse = (double)m * (double)rl.inv_t + ls;
  if (lane == 0) {
    const float hi = some ? (float)lse : -CUDART_INF_F;
    A.out_lse[row] = hi;
    // the two terms are not added first: beside a reference of 1e16 and more ln s would vanish
    if (A.out_tail != nullptr)
      A.out_tail[row] = some && fabsf(hi) < CUDART_INF_F ? (float)(((double)m * (double)rl.inv_t - (double)hi) + ls) : 0.f;
    // an entropy is never negative: the two terms of a row with one likely token may round below
    if (A.out_ent != nullptr) A.out_ent[row] = some ? fmaxf((float)(ls - u / s * (double)rl.inv_t), 0.f) : 0.f;
    if (!some && A.status != nullptr) atomicOr(A.status, 1u);
  }
  for (int g = lane; g < A.G; g += 32) {
    if (g >= 32) gv = score_given<DT>(A, row, rl, g);
    float lp = 0.f;
    if (gv.t >= A.V) {
      lp = -CUDART_INF_F;
      if (A.status != nullptr) atomicOr(A.status, kDevBadToken);
    } else if (gv.t >= 0) {
      lp = some && fabsf(gv.x) < CUDART_INF_F
               ? (float)(((double)gv.x - (double)m) * (double)rl.inv_t - ls)
               : -CUDART_INF_F;
    }
    A.out_lp[row * A.G + g] = lp;
  }
}

__device__ __forceinline__ void score_emit_top(const ScoreArgs& A, long long row, int i, uint32_t key, int idx,
                                               float m, float inv_t, double ls) {
  A.top_ids[row * A.M + i] = idx;
  A.top_lp[row * A.M + i] = (float)(((double)dec_ordered(key) - (double)m) * (double)inv_t - ls);
}
__device__ __forceinline__ void score_emit_no_top(const ScoreArgs& A, long long row, int i) {
  A.top_ids[row * A.M + i] = -1;
  A.top_lp[row * A.M + i] = -CUDART_INF_F;
}

// The row of an emitted position behind the last token.
__device__ __forceinline__ void score_emit_nothing(const ScoreArgs& A, long long row) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) {
    A.out_lse[row] = 0.f;
    if (A.out_ent != nullptr) A.out_ent[row] = 0.f;
    A.out_lp[row] = 0.f;
  }
  for (int i = lane; i < A.M; i += 32) {
    A.top_ids[row * A.M + i] = -1;
    A.top_lp[row * A.M + i] = 0.f;
  }
}

// ------------------------------------------------------------------------------------------
// Many rows: a warp per row.
// ------------------------------------------------------------------------------------------
constexpr int kScoreCtasPerSM = 16;  // one warp each
constexpr int kRowEntries = 80;      // per lane
constexpr int kRowCap = 512;         // listed entries, candidates
// Alternatives per step beyond which a row's entries are groups: an entry per lane and step gives no bound
// beyond 32 of them (280 rows of 1945 bf16, M = 50: 108 -> 13 us, 4000 of 2000, M = 28: 31 -> 25); with
// fewer the second look at the row does not pay (M = 20: 25 us either way).
constexpr int kFineTop = 24;

struct __align__(16) RowShared {
  uint32_t entry[kRowEntries / 2][32];
  unsigned long long cand[kRowCap];
  uint16_t list[kRowCap];
  SelectShared sel;
  int n_list, n;
};

template <int DT, bool ENT>
__global__ void __launch_bounds__(32, kScoreCtasPerSM) score_rows_kernel(const __grid_constant__ ScoreArgs A) {
  extern __shared__ __align__(16) unsigned char score_smem[];
  RowShared& sh = *(RowShared*)score_smem;  // present when M > 0
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int NG = ScoreCfg<DT>::kGroups;
  constexpr int kStep = ScoreCfg<DT>::kStep;
  typedef Group16<DT> Grp;
  const int lane = threadIdx.x;

  for (long long row = blockIdx.x; row < A.rows; row += gridDim.x) {
    const ScoreRow rl = score_locate<ES>(A, row);
    if (!rl.live) {
      score_emit_nothing(A, row);
      continue;
    }
    const float c2 = rl.inv_t * kLog2e;
    const int mis = (int)((uintptr_t)rl.rowp & 31) / ES;
    const int end = mis + A.V;
    const int n_steps = (end + kStep - 1) / kStep;
    const int es = entry_shift(n_steps, kRowEntries), in_entry = (1 << es) - 1;
    EntryColumn col = {&sh.entry[0][lane], ((n_steps - 1) >> es) + 1};

    Grp nxt[NG];
    score_load<DT>(nxt, rl.rowp, mis, end, 0);
    const ScoreGiven given = score_given<DT>(A, row, rl, lane);
    // the first step's maximum is the sums' reference
    const float mx0 = warp_max(score_max<DT>(nxt));
    ScoreSums sums = {mx0 < CUDART_INF_F ? fmaxf(mx0, kGroupLseFloor) : kGroupLseFloor, 0.f, 0.f};
    bool masked = false;
    float top = -CUDART_INF_F;
#pragma unroll 1
    for (int s = 0; s < n_steps; ++s) {
      Grp g[NG];
#pragma unroll
      for (int q = 0; q < NG; ++q) g[q] = nxt[q];
      if (s + 1 < n_steps) score_load<DT>(nxt, rl.rowp, mis, end, s + 1);
      const float mx = score_max<DT>(g);
      if (A.M > 0) {
        top = (s & in_entry) != 0 ? fmaxf(top, mx) : mx;
        col.put(s >> es, top_entry_bits(top, std::integral_constant<int, DT>()));
      }
      score_step<DT, ENT>(g, mx, c2, sums, masked);
    }

    // ---- combine the lanes ---------------------------------------------------------------------
    float m = warp_max(sums.m);
    double2 a = warp_sum2(sums_at(sums, m, c2));
    if (!sums_stand(a, m)) {
      m = warp_max(careful_max<DT>(rl.rowp, lane, 32, A.V));
      a = make_double2(0.0, 0.0);
      if (m > -CUDART_INF_F) a = warp_sum2(careful_sums<DT>(rl.rowp, lane, 32, A.V, m, c2));
    }
    const double ls = a.x > 0.0 ? log(a.x) : 0.0;
    score_emit<DT>(A, row, rl, given, m, a.x, a.y, ls);
    if (A.M == 0) continue;

    // ---- alternatives ----------------------------------------------------------------------------
    int lg = es + (NG == 4 ? 2 : 1);  // log2 of the groups per entry
    if (A.M > kFineTop * n_steps) {
      // few entries, the bound would be loose or none: the short row again, an entry per group
      static_assert((kScoreMaxM / kFineTop + 1) * 4 <= kRowEntries, "the groups' entries fit");
      lg = 0;
      col.n = n_steps * NG;
      for (int s = 0; s < n_steps; ++s) {
        score_load<DT>(nxt, rl.rowp, mis, end, s);
#pragma unroll
        for (int q = 0; q < NG; ++q)
          col.put(s * NG + q, top_entry_bits(score_group_max<DT>(nxt[q]), std::integral_constant<int, DT>()));
      }
    }
    if (col.n & 1) col.put(col.n, 0xff80u);
    if (lane == 0) sh.n_list = sh.n = 0;
    __syncwarp();
    const EntryTest test = entry_test(entry_bound(col, A.M));
    entry_list<kRowEntries / 2>(col, test, sh.list, kRowCap, &sh.n_list, 0);
    __syncwarp();
    if (sh.n_list <= kRowCap) {
      // The listed groups come through shared memory (the entries' place), as many at a time as fit: all
      // of them are on their way together, and the sweep's registers stay what they are.
      constexpr int kPer = (int)sizeof(sh.entry) / (32 * (int)sizeof(Grp));  // groups per lane and turn
      Grp* const stage = (Grp*)&sh.entry[0][0] + lane;
      const int groups = sh.n_list << lg;
      auto where = [&](int i) {
        const int id = sh.list[i >> lg];
        const int g = ((id >> 5) << lg) + (i & ((1 << lg) - 1));
        return g < n_steps * NG ? g * 512 + (id & 31) * 16 : end;
      };
      for (int i0 = lane; i0 < groups; i0 += 32 * kPer) {
        for (int q = 0; q < kPer && i0 + 32 * q < groups; ++q)
          group_fetch<DT>(stage + 32 * q, rl.rowp, where(i0 + 32 * q), mis, end);
        asm volatile("cp.async.wait_all;" ::: "memory");
        for (int q = 0; q < kPer && i0 + 32 * q < groups; ++q) {
          const int v = where(i0 + 32 * q);
          if (v < end) group_candidates<DT>(stage + 32 * q, v, mis, end, test.thr, sh.cand, kRowCap, &sh.n);
        }
      }
    }
    __syncwarp();
    if (sh.n_list > kRowCap || sh.n > kRowCap)
      score_select<DT, 32>(sh.sel, sh.cand, &sh.n, rl.rowp, mis, end, 0, 1, A.M, kRowCap);
    const int n = sh.n;
    rank_candidates(sh.cand, n, lane, 32, [&](int rank, unsigned long long c) {
      if (rank < A.M) score_emit_top(A, row, rank, (uint32_t)(c >> 32), (int)~(uint32_t)c, m, rl.inv_t, ls);
    });
    for (int i = n + lane; i < A.M; i += 32) score_emit_no_top(A, row, i);
    __syncwarp();  // the shared memory is free for the next row
  }
}

// ------------------------------------------------------------------------------------------
// Few rows: a cluster of CTAs per row.  The row's steps are dealt to the cluster's warps in turn; the
// CTAs' statistics and their M best tokens meet in the first CTA through distributed shared memory.
// ------------------------------------------------------------------------------------------
// Four warps a CTA, four CTAs an SM: one CTA's selection runs beside the others' loads (1200 rows of
// 152064 tokens: 85 us; with eight warps and two CTAs 95 us.  One row: 11.3 us against 10.5).
constexpr int kClWarps = 4;
constexpr int kClThreads = 32 * kClWarps;
constexpr int kClCtasPerSM = 16 / kClWarps;
constexpr int kClMaxCtas = 8;       // CTAs per cluster
constexpr int kClEntries = 32;      // per lane
constexpr int kClList = 256 * kClWarps;       // listed entries of a CTA
constexpr int kClCand = 1024;       // tokens of a CTA that reach the bound
static_assert(kClMaxCtas <= 32, "a lane per part");

struct __align__(16) ClusterShared {
  uint32_t entry[kClWarps][kClEntries / 2][32];
  unsigned long long cand[kClCand];
  unsigned long long best[kClMaxCtas][kScoreMaxM];  // the CTAs' M best, in descending order
  uint16_t list[kClList];
  SelectShared sel;
  uint32_t bound[kClWarps];  // at least `share` tokens of the warp have this code or more
  int all_best[kClMaxCtas];  // per CTA of the cluster, in the first one: codes in best, sums, reference
  double2 all_part[kClMaxCtas];
  float all_m[kClMaxCtas];
  float red[kClWarps];
  double2 red2[kClWarps];
  int n_list, n;
};

__device__ __forceinline__ uint32_t cluster_map(const void* p, uint32_t rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t cluster_ld32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_st64(uint32_t a, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_st32(uint32_t a, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
template <int DT, bool ENT>
__global__ void __launch_bounds__(kClThreads, kClCtasPerSM)
score_cluster_kernel(const __grid_constant__ ScoreArgs A, int ctas) {
  extern __shared__ __align__(16) unsigned char score_smem[];
  ClusterShared& sh = *(ClusterShared*)score_smem;
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int NG = ScoreCfg<DT>::kGroups;
  constexpr int kStep = ScoreCfg<DT>::kStep;
  typedef Group16<DT> Grp;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)(blockIdx.x % ctas);
  const long long row = blockIdx.x / ctas;
  const ScoreRow rl = score_locate<ES>(A, row);
  if (ctas > 1) cluster_arrive();  // this CTA has started: its shared memory may be written
  if (!rl.live) {  // the whole cluster
    if (rank == 0 && warp == 0) score_emit_nothing(A, row);
    if (ctas > 1) cluster_wait();
    return;
  }
  const float c2 = rl.inv_t * kLog2e;
  const int mis = (int)((uintptr_t)rl.rowp & 31) / ES;
  const int end = mis + A.V;
  const int n_steps = (end + kStep - 1) / kStep;
  // Many steps: a CTA's warps take neighbouring ones (600 rows of 128256: 52 us, 55 dealt the other way); few:
  // they go to the CTAs in turn, so that the CTAs' shares differ by one at most.
  const int stride = ctas * kClWarps;
  const bool few = n_steps < 2 * stride;
  const int per_warp = few ? ctas : 1, per_rank = few ? 1 : kClWarps;
  const int first = warp * per_warp + rank * per_rank;
  const int mine = first < n_steps ? (n_steps - 1 - first) / stride + 1 : 0;  // steps of this warp
  const int es = entry_shift((n_steps - 1) / stride + 1, kClEntries), in_entry = (1 << es) - 1;
  EntryColumn col = {&sh.entry[warp][0][lane], mine > 0 ? ((mine - 1) >> es) + 1 : 0};

  if (tid == 0) sh.n_list = sh.n = 0;
  Grp nxt[NG];
  ScoreSums sums = {kGroupLseFloor, 0.f, 0.f};
  bool masked = false;
  float top = -CUDART_INF_F;
  ScoreGiven given = {-1, 0.f};
  // the last warp merges the sums and writes the row's outputs while the others rank
  constexpr int kLast = kClWarps - 1;
  if (rank == 0 && warp == kLast) given = score_given<DT>(A, row, rl, lane);
  if (mine > 0) {
    score_load<DT>(nxt, rl.rowp, mis, end, first);
    const float mx0 = warp_max(score_max<DT>(nxt));
    if (mx0 < CUDART_INF_F) sums.m = fmaxf(mx0, kGroupLseFloor);
  }
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    Grp g[NG];
#pragma unroll
    for (int q = 0; q < NG; ++q) g[q] = nxt[q];
    if (i + 1 < mine) score_load<DT>(nxt, rl.rowp, mis, end, first + (i + 1) * stride);
    const float mx = score_max<DT>(g);
    if (A.M > 0) {
      top = (i & in_entry) != 0 ? fmaxf(top, mx) : mx;
      col.put(i >> es, top_entry_bits(top, std::integral_constant<int, DT>()));
    }
    score_step<DT, ENT>(g, mx, c2, sums, masked);
  }
  // Warps of this CTA that have a step, a whole one if any has; each vouches for `share` tokens at or above
  // its own bound, so that M tokens of the row are at or above the smallest of them.  (The row's last step
  // may hold fewer groups than a share: 90 rows of 12420, M = 50, 31 -> 15 us.)
  const int whole = few ? min(kClWarps, (max(0, end / kStep - rank) + ctas - 1) / ctas) : kClWarps;
  const int busy = whole > 0 ? whole : min(kClWarps, (max(0, n_steps - rank) + ctas - 1) / ctas);
  if (A.M > 0 && mine > 0) {
    if (col.n & 1) col.put(col.n, 0xff80u);
  }
  if (A.M > 0 && warp < busy) {
    const uint32_t b = entry_bound(col, (A.M + busy - 1) / busy);
    if (lane == 0) sh.bound[warp] = b;
  }
  {
    const float m = warp_max(sums.m);
    const double2 a = warp_sum2(sums_at(sums, m, c2));
    if (lane == 0) {
      sh.red[warp] = m;
      sh.red2[warp] = a;
    }
  }
  __syncthreads();

  // ---- this CTA's M best and sums go to the cluster's first CTA -----------------------------------
  uint32_t home = (uint32_t)__cvta_generic_to_shared(&sh);
  if (ctas > 1) {
    cluster_wait();
    home = cluster_map(&sh, 0u);
  }
  const uint32_t o_best = (uint32_t)offsetof(ClusterShared, best) + (uint32_t)rank * kScoreMaxM * 8u;
  if (A.M > 0) {
    uint32_t bound = 0xffffffffu;
    for (int w = 0; w < busy; ++w) bound = min(bound, sh.bound[w]);
    const EntryTest test = entry_test(bound);
    if (mine > 0) entry_list<kClEntries / 2>(col, test, sh.list, kClList, &sh.n_list, warp * (kClEntries * 32));
    __syncthreads();
    const int listed = sh.n_list;
    if (listed <= kClList) {
      static_assert(sizeof(sh.entry) >= kClThreads * sizeof(Group16<kF32>), "a group per thread");
      Grp* const stage = (Grp*)&sh.entry[0][0][0] + tid;  // all entries have been listed
      for (int i = tid; i < (listed << es) * NG; i += kClThreads) {
        const int id = sh.list[i / NG >> es];
        const int k = ((id >> 5) % kClEntries << es) + (i / NG & in_entry);  // the warp's k-th step
        const int step = id / (kClEntries * 32) * per_warp + rank * per_rank + k * stride;
        const int v = step * kStep + (i % NG) * 512 + (id & 31) * 16;
        if (step < n_steps && v < end) {
          group_fetch<DT>(stage, rl.rowp, v, mis, end);
          asm volatile("cp.async.wait_all;" ::: "memory");
          group_candidates<DT>(stage, v, mis, end, test.thr, sh.cand, kClCand, &sh.n);
        }
      }
    }
    __syncthreads();
    if (listed > kClList || sh.n > kClCand)
      score_select<DT, kClThreads>(sh.sel, sh.cand, &sh.n, rl.rowp, mis, end, first, stride, A.M, kClCand);
    const int n = sh.n;
    rank_candidates(sh.cand, n, tid, kClThreads, [&](int r, unsigned long long c) {
      if (r < A.M) cluster_st64(home + o_best + 8u * r, c);
    });
    if (tid == 0) cluster_st32(home + (uint32_t)offsetof(ClusterShared, all_best) + 4u * rank, (uint32_t)min(n, A.M));
  }
  if (warp == kLast) {
    const bool on = lane < kClWarps && sh.red2[lane < kClWarps ? lane : 0].x > 0.0;
    const float mw = on ? sh.red[lane] : -CUDART_INF_F;
    // a warp whose sums are NaN spoils the CTA's: the row is then summed again with every check
    const bool odd = lane < kClWarps && !(sh.red2[lane < kClWarps ? lane : 0].x >= 0.0);
    const float m = warp_max(mw);
    double2 a = make_double2(0.0, 0.0);
    if (on) a = part_at(sh.red2[lane], mw, m, c2);
    a = warp_sum2(a);
    if (__any_sync(0xffffffffu, odd)) a.x = CUDART_NAN;
    if (lane == 0) {
      const uint32_t o_part = (uint32_t)offsetof(ClusterShared, all_part) + 16u * rank;
      cluster_st64(home + o_part, (unsigned long long)__double_as_longlong(a.x));
      cluster_st64(home + o_part + 8u, (unsigned long long)__double_as_longlong(a.y));
      cluster_st32(home + (uint32_t)offsetof(ClusterShared, all_m) + 4u * rank, __float_as_uint(m));
    }
  }
  if (ctas > 1) {
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
  }
  __syncthreads();

  // ---- the row -----------------------------------------------------------------------------------
  const float mc = lane < ctas ? sh.all_m[lane] : -CUDART_INF_F;
  float m = warp_max(mc);  // every warp for itself
  double2 a = make_double2(0.0, 0.0);
  if (lane < ctas) {
    if (!(sh.all_part[lane].x >= 0.0)) a.x = CUDART_NAN;
    else if (mc > -CUDART_INF_F) a = part_at(sh.all_part[lane], mc, m, c2);
  }
  a = warp_sum2(a);
  if (!sums_stand(a, m)) {  // uniform over the CTA
    const float mt = warp_max(careful_max<DT>(rl.rowp, tid, kClThreads, A.V));
    __syncthreads();
    if (lane == 0) sh.red[warp] = mt;
    __syncthreads();
    m = sh.red[0];
    for (int w = 1; w < kClWarps; ++w) m = fmaxf(m, sh.red[w]);
    a = make_double2(0.0, 0.0);
    if (m > -CUDART_INF_F) {
      const double2 at = warp_sum2(careful_sums<DT>(rl.rowp, tid, kClThreads, A.V, m, c2));
      if (lane == 0) sh.red2[warp] = at;
      __syncthreads();
      for (int w = 0; w < kClWarps; ++w) {
        a.x += sh.red2[w].x;
        a.y += sh.red2[w].y;
      }
    }
  }
  const double ls = a.x > 0.0 ? log(a.x) : 0.0;  // every warp for itself
  if (warp == kLast) score_emit<DT>(A, row, rl, given, m, a.x, a.y, ls);
  if (A.M == 0) return;
  int total = 0;
  for (int c = 0; c < ctas; ++c) total += sh.all_best[c];
  const int half = 1 << (31 - __clz(A.M));  // the largest power of two that is not above M
  for (int c = warp; c < ctas; c += kClWarps) {
    for (int i = lane; i < sh.all_best[c]; i += 32) {
      const unsigned long long mine = sh.best[c][i];
      // the lists are in descending order: a code's rank is its place in its own list and where it
      // would stand in each other one, found in all of them at once
      int lo[kClMaxCtas], n[kClMaxCtas];
#pragma unroll
      for (int o = 0; o < kClMaxCtas; ++o) {
        lo[o] = 0;
        n[o] = o < ctas && o != c ? sh.all_best[o] : 0;
      }
      for (int bit = ctas > 1 ? half : 0; bit > 0; bit >>= 1) {
#pragma unroll
        for (int o = 0; o < kClMaxCtas; ++o) {
          const int at = lo[o] + bit;
          const unsigned long long other = sh.best[o][min(at, kScoreMaxM) - 1];
          lo[o] = (at <= n[o]) & (other > mine) ? at : lo[o];
        }
      }
      int r = i;
#pragma unroll
      for (int o = 0; o < kClMaxCtas; ++o) r += lo[o];
      if (r < A.M) score_emit_top(A, row, r, (uint32_t)(mine >> 32), (int)~(uint32_t)mine, m, rl.inv_t, ls);
    }
  }
  for (int i = total + tid; i < A.M; i += kClThreads) score_emit_no_top(A, row, i);
}

// ------------------------------------------------------------------------------------------
// Gradient.  With a = g_lse - sum of the gradients of the log probabilities that count,
//     dx_i = (1/T) [ p_i (a - g_H (ln p_i + H)) + sum of the gradients given for token i ].
// A log probability counts when its token is in range and its logit finite.  Masked logits get 0.
// ------------------------------------------------------------------------------------------
struct ScoreGradArgs {
  const void* data;
  long long sb, sk, sj;
  void* grad;
  long long gb, gk, gj;
  int K, J, V, M, G;
  long long rows;
  int chunks, iters;       // chunks per row; a chunk is iters times 64 bytes per thread
  const int32_t* tokens;   // [rows][G]
  const int32_t* top_ids;  // [rows][M]
  const float* lse;        // [rows]
  const float* tail;       // NULL or [rows]
  const float* ent;        // [rows] when g_ent is given
  const float* g_lp;       // NULL or [rows][G]
  const float* g_lse;      // NULL or [rows]
  const float* g_ent;      // NULL or [rows]
  const float* g_top;      // NULL or [rows][M]
  float inv_t[kMaxK], temp[kMaxK];  // 1 / T and T
};

constexpr int kGradThreads = 256;
constexpr int kGradVecs = 2;      // 32-byte vectors per thread, requested together
constexpr int kGradCtasPerSM = 4;

__device__ __forceinline__ void st_stream32(void* p, const Words8& v) {
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v.w[0]),
               "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7])
               : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int DT>
__device__ __forceinline__ void store_elem(char* rowp, long long t, float v) {
  if (DT == kF32)
    ((float*)rowp)[t] = v;
  else
    ((unsigned short*)rowp)[t] = (unsigned short)(pack_bf16x2(v, 0.f) & 0xffffu);
}
// Constants of a row: the gradient at logit x is p (a + b t) with p = 2^t, t = (x - xr) c2 + k.
// xr = lse T as a float; the difference x - xr is taken first and k holds what xr rounded away, so
// that t is good to 2^-23 of its own size however large the logits are.
struct GradRow {
  float xr, c2, k, a, b, inv_t;
  int careful;  // every element is checked by itself (see where it is set); 2: the gradient is 0
};
template <bool ENT>
__device__ __forceinline__ float grad_one(const GradRow& r, float x) {
  if (!(fabsf(x) < CUDART_INF_F)) return 0.f;
  const float t = fmaf(x - r.xr, r.c2, r.k);
  const float p = ex2_approx(t);
  if (!ENT) return p * r.a;
  return p > 0.f ? p * fmaf(r.b, t, r.a) : 0.f;
}

// One 32-byte vector of logits -> gradients (unrounded pairs rounded once into the output type).
template <bool ENT>
__device__ __forceinline__ unsigned long long grad_pair(unsigned long long d2, unsigned long long c22,
                                                        unsigned long long k2, unsigned long long a2,
                                                        unsigned long long b2) {
  const unsigned long long t2 = fma_f32x2(d2, c22, k2);
  float t0, t1;
  unpack_f32x2(t2, t0, t1);
  const unsigned long long p2 = pack_f32x2(ex2_approx(t0), ex2_approx(t1));
  return mul_f32x2(p2, ENT ? fma_f32x2(b2, t2, a2) : a2);
}
template <int DT, bool ENT>
__device__ __forceinline__ void grad_vec(Words8& w, const GradRow& r, float xlow) {
  const unsigned long long c22 = pack_f32x2(r.c2, r.c2), k2 = pack_f32x2(r.k, r.k);
  const unsigned long long a2 = pack_f32x2(r.a, r.a), b2 = pack_f32x2(r.b, r.b);
  const unsigned long long nx2 = pack_f32x2(-r.xr, -r.xr);
  if constexpr (DT == kBF16) {
    Group16<kBF16> g;
    g.a = w;
    if (r.careful || group16_max(g) == CUDART_INF_F) {
#pragma unroll
      for (int t = 0; t < 8; ++t)
        w.w[t] = pack_bf16x2(grad_one<ENT>(r, bf16_lo(w.w[t])), grad_one<ENT>(r, bf16_hi(w.w[t])));
      return;
    }
    // logits so low that p is 0 whatever they are, -inf and NaN all become the same low value
    const uint32_t low = bf16_floor_bits(xlow) * 0x10001u;
#pragma unroll
    for (int t = 0; t < 8; ++t) g.a.w[t] = max_bf16x2(g.a.w[t], low);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      float o0, o1;
      unpack_f32x2(grad_pair<ENT>(group16_diff2(g, 2 * t, -r.xr, nx2), c22, k2, a2, b2), o0, o1);
      w.w[t] = pack_bf16x2(o0, o1);
    }
  } else {
    float mx = -CUDART_INF_F;
#pragma unroll
    for (int t = 0; t < 8; ++t) mx = fmaxf(mx, __uint_as_float(w.w[t]));
    if (r.careful || mx == CUDART_INF_F) {
#pragma unroll
      for (int t = 0; t < 8; ++t) w.w[t] = __float_as_uint(grad_one<ENT>(r, __uint_as_float(w.w[t])));
      return;
    }
#pragma unroll
    for (int t = 0; t < 8; t += 2) {
      const unsigned long long d2 =
          add_f32x2(pack_f32x2(fmaxf(__uint_as_float(w.w[t]), xlow), fmaxf(__uint_as_float(w.w[t + 1]), xlow)), nx2);
      float o0, o1;
      unpack_f32x2(grad_pair<ENT>(d2, c22, k2, a2, b2), o0, o1);
      w.w[t] = __float_as_uint(o0);
      w.w[t + 1] = __float_as_uint(o1);
    }
  }
}

// The given tokens and alternatives of a row, one after the other.
struct GradEntry {
  int t;
  float g;
};
__device__ __forceinline__ GradEntry grad_entry(const ScoreGradArgs& A, long long row, int n_lp, int e) {
  GradEntry r;
  if (e < n_lp) {
    r.t = __ldg(A.tokens + row * A.G + e);
    r.g = __ldg(A.g_lp + row * A.G + e);
  } else {
    r.t = __ldg(A.top_ids + row * A.M + (e - n_lp));
    r.g = __ldg(A.g_top + row * A.M + (e - n_lp));
  }
  return r;
}

// A CTA takes chunks of rows in turn.  Each warp forms the row's constants for itself while its first
// loads are in flight (no barrier: waiting for one thread's constants took half of the kernel's time),
// writes its gradients, and the thread that wrote a given token's element writes it again with the
// extra term (added in fp32 before the one rounding; a token given twice is written once, with the
// sum taken in the order given).
template <int DT, bool ENT>
__global__ void __launch_bounds__(kGradThreads, kGradCtasPerSM) score_grad_kernel(const __grid_constant__ ScoreGradArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int EV = 32 / ES;                           // elements per vector
  constexpr int kTurn = kGradThreads * kGradVecs * EV;  // elements per turn of the CTA
  const int tid = threadIdx.x, lane = tid & 31;
  const long long n_items = A.rows * A.chunks;
  const int n_lp = A.g_lp != nullptr ? A.G : 0;
  const int n_e = n_lp + (A.g_top != nullptr ? A.M : 0);
  for (long long it = blockIdx.x; it < n_items; it += gridDim.x) {
    const uint32_t row = n_items < (1ll << 32) ? (uint32_t)it / (uint32_t)A.chunks : (uint32_t)(it / A.chunks);
    const int chunk = (int)(it - (long long)row * A.chunks);
    const uint32_t bk = row / (uint32_t)A.J, b = bk / (uint32_t)A.K;
    const int j = (int)(row - bk * (uint32_t)A.J), k = (int)(bk - b * (uint32_t)A.K);
    const char* const rowp = (const char*)A.data + (b * A.sb + k * A.sk + j * A.sj) * ES;
    char* const outp = (char*)A.grad + (b * A.gb + k * A.gk + j * A.gj) * ES;
    const int mis = (int)((uintptr_t)rowp & 31) / ES;
    const bool same = ((uintptr_t)rowp & 31) == ((uintptr_t)outp & 31);
    const int end = mis + A.V;
    const long long first = (long long)chunk * A.iters * kTurn + tid * EV;  // this thread's first vector

    Words8 w[kGradVecs];
    auto load = [&](int q, long long v) {
      if (v >= mis && v + EV <= end) w[q] = ld_stream32(rowp + (v - mis) * ES);
    };
#pragma unroll
    for (int q = 0; q < kGradVecs; ++q) load(q, first + q * (kGradThreads * EV));

    // ---- the row's constants -----------------------------------------------------------------------
    GradRow r;
    r.inv_t = A.inv_t[k];
    r.c2 = r.inv_t * kLog2e;
    {
      const float lse = __ldg(A.lse + row);
      const float tail = A.tail != nullptr ? __ldg(A.tail + row) : 0.f;
      float gh = 0.f, h = 0.f;
      if (ENT) {
        gh = __ldg(A.g_ent + row);
        h = __ldg(A.ent + row);
      }
      float a = A.g_lse != nullptr ? __ldg(A.g_lse + row) : 0.f;
      if (n_e > 0) {
        double sum = 0.0;
        for (int e = lane; e < n_e; e += 32) {
          const GradEntry ge = grad_entry(A, row, n_lp, e);
          if (ge.t >= 0 && ge.t < A.V && fabsf(load_logit<DT>(rowp, ge.t)) < CUDART_INF_F) sum += (double)ge.g;
        }
        if (n_e > 1) {
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        } else {
          sum = __shfl_sync(0xffffffffu, sum, 0);
        }
        a = (float)((double)a - sum);
      }
      if (ENT) a = fmaf(-gh, h, a);
      r.a = a * r.inv_t;
      r.b = ENT ? -gh * (0.69314718056f * r.inv_t) : 0.f;  // ln p = t ln 2
      r.xr = lse * A.temp[k];
      if (fabsf(lse) < CUDART_INF_F && fabsf(r.xr) < CUDART_INF_F) {
        r.k = (float)((((double)r.xr * (double)r.inv_t - (double)lse) - (double)tail) * 1.4426950408889634074);
        // logits beyond 1e30 in size, or a temperature so low that xr - 200 / c2 could round to xr
        r.careful = fabsf(r.xr) >= 1e30f || fabsf(r.xr) * r.c2 > 1e8f;
      } else {  // a row without a finite logit has no gradient
        r.xr = r.a = r.b = 0.f;
        r.k = -CUDART_INF_F;
        r.careful = 2;
      }
    }
    const float xlow = r.xr - 200.0f / r.c2;

    for (int i = 0; i < A.iters; ++i) {
      const long long v0 = first + (long long)i * kTurn;
      if (v0 - lane * EV >= end) break;
#pragma unroll
      for (int q = 0; q < kGradVecs; ++q) {
        const long long v = v0 + q * (kGradThreads * EV);
        if (v >= mis && v + EV <= end) {
          grad_vec<DT, ENT>(w[q], r, xlow);
          char* const o = outp + (v - mis) * ES;
          if (same) {
            st_stream32(o, w[q]);
          } else {
#pragma unroll
            for (int t = 0; t < EV; ++t) {
              if (DT == kF32)
                ((float*)o)[t] = __uint_as_float(w[q].w[t % 8]);
              else
                ((unsigned short*)o)[t] = (unsigned short)(w[q].w[t / 2] >> (16 * (t & 1)));
            }
          }
        }
        if (i + 1 < A.iters) load(q, v + kTurn);  // the next turn's, as soon as the registers are free
      }
    }
    // the vectors that stick out of the row at its ends: an element per thread
    const long long c0 = (long long)chunk * A.iters * kTurn;
    if (tid < EV) {
      auto edge = [&](long long v) {
        if (v >= mis && v < end) store_elem<DT>(outp, v - mis, grad_one<ENT>(r, load_logit<DT>(rowp, v - mis)));
      };
      const long long tail = (long long)end / EV * EV;  // starts the last vector when that is not full
      if (chunk == 0 && (mis > 0 || end < EV)) edge(tid);
      if (tail < end && tail > 0 && tail >= c0 && tail < c0 + (long long)A.iters * kTurn) edge(tail + tid);
    }

    // ---- the given tokens' own elements, by the threads that have just written them -----------------
    for (int e = 0; e < n_e; ++e) {
      const GradEntry ge = grad_entry(A, row, n_lp, e);
      const long long v = (long long)ge.t + mis, vec = v / EV * EV;
      if (ge.t < 0 || ge.t >= A.V || vec < c0 || vec >= c0 + (long long)A.iters * kTurn || r.careful == 2) continue;
      const bool whole = vec >= mis && vec + EV <= end;
      if ((whole ? (int)((vec - c0) / EV % kGradThreads) : (int)(v - vec)) != tid) continue;
      const float x = load_logit<DT>(rowp, ge.t);
      if (!(fabsf(x) < CUDART_INF_F)) continue;
      double g = 0.0;
      bool given_before = false;
      for (int o = 0; o < n_e; ++o) {
        const GradEntry other = grad_entry(A, row, n_lp, o);
        if (other.t != ge.t) continue;
        if (o < e) given_before = true;
        g += (double)other.g;
      }
      if (!given_before) store_elem<DT>(outp, ge.t, fmaf((float)g, r.inv_t, grad_one<ENT>(r, x)));
    }
  }
}

}  // namespace gls
