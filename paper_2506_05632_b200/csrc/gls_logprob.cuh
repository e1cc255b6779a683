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
#include "gls_topm.cuh"

namespace gls {

constexpr int kScoreMaxM = kTopmMaxM;    // alternatives per row
constexpr int kScoreMaxG = 64;           // given tokens per row
constexpr int kScoreMaxCand = 4096;      // candidates of all slices of a row that the merge sorts
constexpr int kScoreCtasPerSM = 16;      // one warp each
constexpr uint32_t kDevBadToken = 2u;    // GLS_DEV_BAD_TOKEN

// Softmax statistics of one slice of a row: sums relative to the reference logit m.
// s == 0: the slice has no finite logit.
struct __align__(16) ScorePart {
  float m, s, u;
  int n;  // candidates the slice left
};

struct ScoreArgs {
  const void* data;       // rows [B][K][J][V]
  long long sb, sk, sj;   // element strides
  int K, J, V, M, G;
  int emitted;            // 1: row (b, j) is that of the lowest draft active at j (see accept)
  int L;
  const uint8_t* accept;  // [B][K][L]
  long long rows;         // B * K * J, or B * J for emitted rows
  int splits, steps_per_slice;
  const int32_t* tokens;  // [rows][G]
  float inv_t[kMaxK];
  float* out_lp;          // [rows][G]
  float* out_lse;         // [rows]
  float* out_tail;        // NULL or [rows]: lse - out_lse in the precision that fp32 leaves
  float* out_ent;         // NULL or [rows]
  int32_t* top_ids;       // [rows][M]
  float* top_lp;          // [rows][M]
  ScorePart* parts;       // [rows][splits]
  unsigned long long* cand;  // [rows][splits][M]: (ordered code << 32) | ~index
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
  const int j = (int)(row % A.J);
  if (A.emitted) {
    b = row / A.J;
    k = 0;
    r.live = __ldg(A.tokens + row) >= 0;
    if (r.live && j > 0) {  // lowest draft whose position j - 1 was accepted
      const uint8_t* a = A.accept + b * A.K * A.L + (j - 1);
      const unsigned lo = __ballot_sync(0xffffffffu, lane < A.K && a[(long long)lane * A.L] != 0);
      const unsigned hi = __ballot_sync(0xffffffffu, lane + 32 < A.K && a[(long long)(lane + 32) * A.L] != 0);
      k = lo != 0u ? __ffs(lo) - 1 : hi != 0u ? 31 + __ffs(hi) : 0;
    }
  } else {
    const long long bk = row / A.J;
    k = (int)(bk % A.K);
    b = bk / A.K;
    r.live = true;
  }
  r.inv_t = A.inv_t[k];
  r.rowp = (const char*)A.data + (b * A.sb + (long long)k * A.sk + (long long)j * A.sj) * ES;
  return r;
}

template <int DT>
struct ScoreCfg {  // one step of a warp: 4 KB of the row
  static constexpr int kGroups = DT == kBF16 ? 4 : 2;  // groups of 16 tokens per lane
  static constexpr int kStep = 512 * kGroups;
};

__device__ __forceinline__ unsigned long long score_code(uint32_t key, int idx) {
  return ((unsigned long long)key << 32) | (uint32_t)~idx;
}

// The largest float below x (x finite).
__device__ __forceinline__ float just_below(float x) {
  const uint32_t b = __float_as_uint(x);
  if (x == 0.f) return __uint_as_float(0x80000001u);
  return __uint_as_float(x > 0.f ? b - 1u : b + 1u);
}

// Examines queued groups (indices of 16-token groups counted from the 32-byte boundary at or below
// the row's start, `mis` elements before it): appends their tokens above thr to the buffer in index
// order and prunes it past M + 64 entries.  Returns (threshold bits << 32) | new count.
template <int DT>
__device__ __noinline__ unsigned long long score_expand(TopmWarpBuf* wb, const int* queue, const char* rowp,
                                                        int mis, int V, int first, int nb, int n, int M,
                                                        float thr) {
  const int lane = threadIdx.x & 31;
  float a[16];
  uint32_t m = 0u;
  int tok = 0;
  if (lane < nb) {
    tok = (queue[first + lane] << 4) - mis;
#pragma unroll
    for (int t = 0; t < 16; ++t)
      a[t] = tok + t >= 0 && tok + t < V ? load_logit<DT>(rowp, tok + t) : -CUDART_INF_F;
#pragma unroll
    for (int t = 0; t < 16; ++t)
      if (a[t] > thr && a[t] < CUDART_INF_F) m |= 1u << t;  // false for NaN
  }
  const int cnt = __popc(m);
  int incl = cnt;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  int pos = n + incl - cnt;
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    if ((m >> t) & 1u) {
      if (GLS_IN_RANGE(pos, 0, kTopmCap, 60u)) {
        wb->key[pos] = enc_ordered(a[t] + 0.0f);  // -0 and +0 are the same logit: one code
        wb->idx[pos] = tok + t;
      }
      ++pos;
    }
  }
  n += __shfl_sync(0xffffffffu, incl, 31);
  __syncwarp();
  if (n > M + 64) {
    const unsigned long long r = topm_prune(wb, n, M, DT == kBF16 ? 2 : 0);
    n = (int)(unsigned)r;
    thr = dec_ordered((uint32_t)(r >> 32));
  }
  return ((unsigned long long)__float_as_uint(thr) << 32) | (unsigned)n;
}

// Statistics of tokens [t0, t1) of a row with every element checked, two passes, sums in 64 bits:
// for slices on which the sweep's arithmetic does not hold (NaN or +inf logits, logits beyond 1e30
// in size, no finite logit at all).  Warp-collective; every lane returns the result.
template <int DT>
__device__ __noinline__ ScorePart score_careful(const char* rowp, int t0, int t1, float c2) {
  const int lane = threadIdx.x & 31;
  float m = -CUDART_INF_F;
  for (int t = t0 + lane; t < t1; t += 32) {
    const float x = load_logit<DT>(rowp, t);
    if (fabsf(x) < CUDART_INF_F) m = fmaxf(m, x);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  ScorePart r;
  r.m = m;
  r.s = r.u = 0.f;
  r.n = 0;
  if (m == -CUDART_INF_F) return r;
  double s = 0.0, u = 0.0;
  for (int t = t0 + lane; t < t1; t += 32) {
    const float x = load_logit<DT>(rowp, t);
    if (!(fabsf(x) < CUDART_INF_F)) continue;
    const double d = (double)x - (double)m;
    const double e = exp2(d * (double)c2);
    s += e;
    if (e > 0.0) u += e * d;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, d);
    u += __shfl_xor_sync(0xffffffffu, u, d);
  }
  r.s = (float)s;
  r.u = (float)u;
  return r;
}

// Outputs of one row except its alternatives, by one warp.  m reference logit, s and u the sums.
template <int DT>
__device__ __forceinline__ double score_emit(const ScoreArgs& A, long long row, const ScoreRow& rl, float m,
                                             double s, double u) {
  const int lane = threadIdx.x & 31;
  const bool some = s > 0.0;
  const double ls = some ? log(s) : 0.0;
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
    const int t = __ldg(A.tokens + row * A.G + g);
    float lp = 0.f;
    if (t >= A.V) {
      lp = -CUDART_INF_F;
      if (A.status != nullptr) atomicOr(A.status, kDevBadToken);
    } else if (t >= 0) {
      const float x = load_logit<DT>(rl.rowp, t);
      lp = some && fabsf(x) < CUDART_INF_F
               ? (float)(((double)x - (double)m) * (double)rl.inv_t - ls)
               : -CUDART_INF_F;
    }
    A.out_lp[row * A.G + g] = lp;
  }
  return ls;
}

__device__ __forceinline__ void score_emit_top(const ScoreArgs& A, long long row, int i, uint32_t key, int idx,
                                               float m, float inv_t, double ls) {
  A.top_ids[row * A.M + i] = idx;
  A.top_lp[row * A.M + i] = (float)(((double)dec_ordered(key) - (double)m) * (double)inv_t - ls);
}

// The row of an emitted position behind the last token.
__device__ __forceinline__ void score_emit_nothing(const ScoreArgs& A, long long row) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) {
    A.out_lse[row] = 0.f;
    if (A.out_tail != nullptr) A.out_tail[row] = 0.f;
    if (A.out_ent != nullptr) A.out_ent[row] = 0.f;
    A.out_lp[row] = 0.f;
  }
  for (int i = lane; i < A.M; i += 32) {
    A.top_ids[row * A.M + i] = -1;
    A.top_lp[row * A.M + i] = 0.f;
  }
}

// One pass over the rows.  A warp takes (row, slice) items in turn.
template <int DT, bool ENT>
__global__ void __launch_bounds__(32, kScoreCtasPerSM) score_kernel(const __grid_constant__ ScoreArgs A) {
  extern __shared__ __align__(16) unsigned char score_smem[];
  TopmWarpBuf* const wb = (TopmWarpBuf*)score_smem;  // present when M > 0
  __shared__ int queue[kS4QueueCap];
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int NG = ScoreCfg<DT>::kGroups;
  constexpr int kStep = ScoreCfg<DT>::kStep;
  typedef Group16<DT> Grp;
  const int lane = threadIdx.x & 31;
  const uint32_t lt = (1u << lane) - 1u;
  const long long n_items = A.rows * A.splits;

  for (long long it = blockIdx.x; it < n_items; it += gridDim.x) {
    const long long row = it / A.splits;
    const int split = (int)(it % A.splits);
    const ScoreRow rl = score_locate<ES>(A, row);
    if (!rl.live) {
      if (split == 0) score_emit_nothing(A, row);
      continue;
    }
    const float c2 = rl.inv_t * kLog2e;
    // the row in groups counted from the 32-byte boundary at or below its start, so that a row
    // that starts anywhere is read by aligned 32-byte loads; only groups that stick out at either
    // end are read element by element
    const int mis = (int)((uintptr_t)rl.rowp & 31) / ES;
    const char* const base = rl.rowp - mis * ES;
    const int end = mis + A.V;
    const int n_steps = (end + kStep - 1) / kStep;
    const int s_begin = split * A.steps_per_slice;
    const int s_end = min(n_steps, s_begin + A.steps_per_slice);

    auto load_step = [&](Grp (&g)[NG], int s) {
      const int v0 = s * kStep + lane * 16;
#pragma unroll
      for (int q = 0; q < NG; ++q) {
        const int v = v0 + q * 512;
        if (v >= mis && v + 16 <= end) {
          load16_vec(g[q], base + (size_t)v * ES);
        } else {
          float x[16];
#pragma unroll
          for (int t = 0; t < 16; ++t)
            x[t] = v + t >= mis && v + t < end ? load_logit<DT>(rl.rowp, v + t - mis) : -CUDART_INF_F;
          if constexpr (DT == kBF16) {
#pragma unroll
            for (int t = 0; t < 8; ++t)
              g[q].a.w[t] = (__float_as_uint(x[2 * t]) >> 16) | (__float_as_uint(x[2 * t + 1]) & 0xffff0000u);
          } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
              g[q].a.w[t] = __float_as_uint(x[t]);
              g[q].b.w[t] = __float_as_uint(x[8 + t]);
            }
          }
        }
      }
    };

    float thr = A.M > 0 ? -CUDART_INF_F : CUDART_INF_F;
    int n = 0, qn = 0, s = s_begin;
    float lm = kGroupLseFloor;
    float s_tot = 0.f, u_tot = 0.f;
    Grp nxt[NG];
    if (s < s_end) {
      load_step(nxt, s);
      // the first step's maximum is the sums' reference; the M-th largest of its group maxima
      // (distinct tokens) bounds the M-th largest logit of the row from below
      float gm[NG];
      float mx = -CUDART_INF_F;
#pragma unroll
      for (int q = 0; q < NG; ++q) {
        gm[q] = group16_max(nxt[q]);
        if (gm[q] == CUDART_INF_F) gm[q] = -CUDART_INF_F;
        mx = fmaxf(mx, gm[q]);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      lm = fmaxf(lm, mx);
      if (A.M > 0 && A.M <= 32 * NG) {
        uint32_t code[NG], kth = 0u;
#pragma unroll
        for (int q = 0; q < NG; ++q) code[q] = enc_ordered(gm[q] + 0.0f);
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit != 0u; bit >>= 1) {
          int c = 0;
#pragma unroll
          for (int q = 0; q < NG; ++q) c += __popc(__ballot_sync(0xffffffffu, code[q] >= (kth | bit)));
          if (c >= A.M) kth |= bit;
        }
        const float f = dec_ordered(kth);
        if (f > -CUDART_INF_F) thr = just_below(f);
      }
    }
    __syncwarp();
    for (;;) {
#pragma unroll 1
      for (; s < s_end && qn < 32; ++s) {
        Grp g[NG];
#pragma unroll
        for (int q = 0; q < NG; ++q) g[q] = nxt[q];
        if (s + 1 < s_end) load_step(nxt, s + 1);
        unsigned long long s2 = 0ull, u2 = 0ull;  // this step's sums; folded into the totals below
#pragma unroll
        for (int q = 0; q < NG; ++q) {
          const float amax = group16_max(g[q]);
          const bool hit = amax > thr;  // false for NaN
          const unsigned bal = __ballot_sync(0xffffffffu, hit);
          if (bal != 0u) {
            if (hit && GLS_IN_RANGE(qn + __popc(bal & lt), 0, kS4QueueCap, 61u))
              queue[qn + __popc(bal & lt)] = ((s * kStep + q * 512) >> 4) + lane;
            qn += __popc(bal);
          }
          // The reference moves only when a maximum exceeds it by 2^8: the terms stay within
          // fp32 and the two parts of the entropy small.
          if (fmaf(amax - lm, c2, -8.0f) > 0.f && amax < CUDART_INF_F) {
            const float r = ex2_approx((lm - amax) * c2);
            const float dl = lm - amax;  // x - amax = (x - lm) + (lm - amax)
            float s0, s1, u0, u1;
            unpack_f32x2(s2, s0, s1);
            unpack_f32x2(u2, u0, u1);
            if (ENT) {
              u2 = pack_f32x2(r > 0.f ? r * (u0 + s0 * dl) : 0.f, r > 0.f ? r * (u1 + s1 * dl) : 0.f);
              u_tot = r > 0.f ? r * (u_tot + s_tot * dl) : 0.f;
            }
            s2 = pack_f32x2(r * s0, r * s1);
            s_tot *= r;
            lm = amax;
          }
          const unsigned long long c22 = pack_f32x2(c2, c2), nlm2 = pack_f32x2(-lm, -lm);
          Grp h = g[q];
          if (ENT) {
            // -inf and NaN become the lowest finite value: their terms are exactly 0 in both sums
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
            s2 = add_f32x2(s2, e2);
            if (ENT) u2 = fma_f32x2(e2, d2, u2);
          }
        }
        float a0, a1;
        unpack_f32x2(s2, a0, a1);
        s_tot += a0 + a1;
        if (ENT) {
          unpack_f32x2(u2, a0, a1);
          u_tot += a0 + a1;
        }
      }
      if (qn == 0) break;
      __syncwarp();
      for (int first = 0; first < qn; first += 32) {
        const unsigned long long r =
            score_expand<DT>(wb, queue, rl.rowp, mis, A.V, first, min(32, qn - first), n, A.M, thr);
        n = (int)(unsigned)r;
        thr = __uint_as_float((uint32_t)(r >> 32));
      }
      qn = 0;
      __syncwarp();
      if (s >= s_end) break;
    }
    if (n > A.M) n = (int)(unsigned)topm_prune(wb, n, A.M, DT == kBF16 ? 2 : 0);
    __syncwarp();

    // ---- combine the lanes ---------------------------------------------------------------------
    float m = lm;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float r = ex2_approx((lm - m) * c2);
    double sd = (double)s_tot * r;
    double ud = r > 0.f ? ((double)u_tot + (double)s_tot * ((double)lm - (double)m)) * r : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      sd += __shfl_xor_sync(0xffffffffu, sd, d);
      if (ENT) ud += __shfl_xor_sync(0xffffffffu, ud, d);
    }
    // sums that are zero, infinite or NaN, or a reference out of the range in which a difference
    // of two logits can not overflow
    if (!(sd > 0.0 && sd < (double)CUDART_INF_F && fabs(ud) < (double)CUDART_INF_F && m < 1e30f)) {
      const int t0 = max(0, s_begin * kStep - mis);
      const int t1 = (int)min((long long)A.V, (long long)s_end * kStep - mis);
      const ScorePart p = score_careful<DT>(rl.rowp, t0, t1, c2);
      m = p.m;
      sd = p.s;
      ud = p.u;
    }
    if (A.splits == 1) {
      const double ls = score_emit<DT>(A, row, rl, m, sd, ud);
      for (int i = lane; i < A.M; i += 32) {  // rank of entry i: how many come before it
        int rank = i;
        int idx = -1;
        uint32_t key = 0u;
        if (i < n) {
          key = wb->key[i];
          idx = wb->idx[i];
          rank = 0;
          const unsigned long long mine = score_code(key, idx);
          for (int o = 0; o < n; ++o) rank += score_code(wb->key[o], wb->idx[o]) > mine;
        }
        if (idx >= 0) {
          score_emit_top(A, row, rank, key, idx, m, rl.inv_t, ls);
        } else {
          A.top_ids[row * A.M + i] = -1;
          A.top_lp[row * A.M + i] = -CUDART_INF_F;
        }
      }
    } else {
      const long long at = row * A.splits + split;
      if (lane == 0) {
        ScorePart p;
        p.m = m;
        p.s = (float)sd;
        p.u = (float)ud;
        p.n = n;
        A.parts[at] = p;
      }
      for (int i = lane; i < n; i += 32) A.cand[at * A.M + i] = score_code(wb->key[i], wb->idx[i]);
    }
    __syncwarp();  // the buffer is free for the next item
  }
  asm volatile("griddepcontrol.launch_dependents;");
}

// Merges the slices of a row: statistics in 64 bits, the slices' candidates sorted in shared memory.
constexpr int kScoreMergeThreads = 256;
template <int DT>
__global__ void __launch_bounds__(kScoreMergeThreads) score_merge_kernel(const __grid_constant__ ScoreArgs A) {
  extern __shared__ __align__(16) unsigned char score_smem[];
  unsigned long long* const codes = (unsigned long long*)score_smem;
  __shared__ int sh_n;
  __shared__ double sh_ls;
  __shared__ float sh_m;
  constexpr int ES = DT == kBF16 ? 2 : 4;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the sweep's writes are visible
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (long long row = blockIdx.x; row < A.rows; row += gridDim.x) {
    const ScoreRow rl = score_locate<ES>(A, row);
    if (!rl.live) continue;  // uniform over the CTA
    const ScorePart* parts = A.parts + row * A.splits;
    if (tid == 0) sh_n = 0;
    __syncthreads();
    if (warp == 0) {
      const double c2 = (double)(rl.inv_t * kLog2e);
      float m = -CUDART_INF_F;
      for (int i = lane; i < A.splits; i += 32) {
        const ScorePart p = parts[i];
        if (p.s > 0.f) m = fmaxf(m, p.m);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      double s = 0.0, u = 0.0;
      for (int i = lane; i < A.splits; i += 32) {
        const ScorePart p = parts[i];
        if (p.s > 0.f) {
          const double dl = (double)p.m - (double)m;
          const double r = exp2(dl * c2);
          s += r * (double)p.s;
          if (r > 0.0) u += r * ((double)p.u + (double)p.s * dl);
        }
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, d);
        u += __shfl_xor_sync(0xffffffffu, u, d);
      }
      const double ls = score_emit<DT>(A, row, rl, m, s, u);
      if (lane == 0) {
        sh_ls = ls;
        sh_m = m;
      }
    }
    if (A.M > 0) {
      for (int i = warp; i < A.splits; i += kScoreMergeThreads / 32) {
        const int n = parts[i].n;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh_n, n);  // the order does not matter: the codes are sorted
        at = __shfl_sync(0xffffffffu, at, 0);
        for (int o = lane; o < n; o += 32)
          if (GLS_IN_RANGE(at + o, 0, kScoreMaxCand, 62u)) codes[at + o] = A.cand[(row * A.splits + i) * A.M + o];
      }
      __syncthreads();
      const int n = sh_n;
      int p2 = 32;
      while (p2 < n) p2 <<= 1;
      for (int i = n + tid; i < p2; i += kScoreMergeThreads) codes[i] = 0ull;
      __syncthreads();
      for (int size = 2; size <= p2; size <<= 1) {  // bitonic sort, descending
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
          for (int i = tid; i < p2 / 2; i += kScoreMergeThreads) {
            const int a = 2 * i - (i & (stride - 1)), b = a + stride;
            const unsigned long long x = codes[a], y = codes[b];
            if ((x < y) == ((a & size) == 0)) {
              codes[a] = y;
              codes[b] = x;
            }
          }
          __syncthreads();
        }
      }
      for (int i = tid; i < A.M; i += kScoreMergeThreads) {
        if (i < n) {
          const unsigned long long c = codes[i];
          score_emit_top(A, row, i, (uint32_t)(c >> 32), (int)~(uint32_t)c, sh_m, rl.inv_t, sh_ls);
        } else {
          A.top_ids[row * A.M + i] = -1;
          A.top_lp[row * A.M + i] = -CUDART_INF_F;
        }
      }
    }
    __syncthreads();
  }
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
  int chunks;              // chunks per row
  const int32_t* tokens;   // [rows][G]
  const int32_t* top_ids;  // [rows][M]
  const float* lse;        // [rows]
  const float* tail;       // NULL or [rows]
  const float* ent;        // [rows] when g_ent is given
  const float* g_lp;       // NULL or [rows][G]
  const float* g_lse;      // NULL or [rows]
  const float* g_ent;      // NULL or [rows]
  const float* g_top;      // NULL or [rows][M]
  float inv_t[kMaxK];
};

constexpr int kGradThreads = 256;
constexpr int kGradVecs = 4;  // 32-byte vectors per thread and chunk
constexpr int kGradMaxEntries = kScoreMaxG + kScoreMaxM;

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
// x rounded down to bf16 (finite x well inside the range)
__device__ __forceinline__ uint32_t bf16_floor_bits(float x) {
  uint32_t b = __float_as_uint(x);
  if (b & 0x80000000u) b += 0xffffu;
  return b >> 16;
}

// Constants of a row: the gradient at logit x is p (a + b t) with p = 2^t, t = (x - xr) c2 + k.
// xr = lse T as a float; the difference x - xr is taken first and k holds what xr rounded away, so
// that t is good to 2^-23 of its own size however large the logits are.
struct GradRow {
  float xr, c2, k, a, b, inv_t;
  int careful;  // the row's logits are beyond 1e30 in size: every element is checked by itself
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

// A CTA takes chunks of rows in turn: reads the chunk, forms the row's constants while the loads are
// in flight, writes the gradients, then writes the given tokens' own elements again with their
// extra term (added in fp32 before the one rounding; a token given twice is written once, with the
// sum taken in the order given).
template <int DT, bool ENT>
__global__ void __launch_bounds__(kGradThreads) score_grad_kernel(const __grid_constant__ ScoreGradArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int EV = 32 / ES;                            // elements per vector
  constexpr int kChunk = kGradThreads * kGradVecs * EV;  // elements per chunk
  __shared__ int e_tok[kGradMaxEntries];
  __shared__ float e_g[kGradMaxEntries], e_x[kGradMaxEntries];
  __shared__ GradRow sh_row;
  const int tid = threadIdx.x;
  const long long n_items = A.rows * A.chunks;
  const int n_lp = A.g_lp != nullptr ? A.G : 0;
  const int n_e = n_lp + (A.g_top != nullptr ? A.M : 0);
  for (long long it = blockIdx.x; it < n_items; it += gridDim.x) {
    const long long row = it / A.chunks;
    const int chunk = (int)(it % A.chunks);
    const int j = (int)(row % A.J);
    const long long bk = row / A.J;
    const int k = (int)(bk % A.K);
    const long long b = bk / A.K;
    const char* rowp = (const char*)A.data + (b * A.sb + k * A.sk + j * A.sj) * ES;
    char* outp = (char*)A.grad + (b * A.gb + k * A.gk + j * A.gj) * ES;
    const int mis = (int)((uintptr_t)rowp & 31) / ES;
    const bool same = ((uintptr_t)rowp & 31) == ((uintptr_t)outp & 31);
    const int end = mis + A.V;
    const long long v0 = (long long)chunk * kChunk;

    Words8 w[kGradVecs];
#pragma unroll
    for (int q = 0; q < kGradVecs; ++q) {
      const long long v = v0 + (q * kGradThreads + tid) * EV;
      if (v >= mis && v + EV <= end) w[q] = ld_stream32(rowp + (v - mis) * ES);
    }
    for (int e = tid; e < n_e; e += kGradThreads) {
      const int t = e < n_lp ? __ldg(A.tokens + row * A.G + e) : __ldg(A.top_ids + row * A.M + (e - n_lp));
      e_tok[e] = t;
      e_g[e] = e < n_lp ? __ldg(A.g_lp + row * A.G + e) : __ldg(A.g_top + row * A.M + (e - n_lp));
      e_x[e] = t >= 0 && t < A.V ? load_logit<DT>(rowp, t) : -CUDART_INF_F;
    }
    __syncthreads();
    if (tid < 32) {
      double a = 0.0;
      for (int e = tid; e < n_e; e += 32)
        if (fabsf(e_x[e]) < CUDART_INF_F) a -= (double)e_g[e];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
      if (tid == 0) {
        const double inv_t = (double)A.inv_t[k];
        const float lse = __ldg(A.lse + row);
        const double tail = A.tail != nullptr ? (double)__ldg(A.tail + row) : 0.0;
        const double kLog2eD = 1.4426950408889634074;
        GradRow r;
        r.inv_t = A.inv_t[k];
        r.c2 = A.inv_t[k] * kLog2e;
        if (A.g_lse != nullptr) a += (double)__ldg(A.g_lse + row);
        double gb = 0.0;
        if (ENT) {
          const double gh = (double)__ldg(A.g_ent + row);
          a -= gh * (double)__ldg(A.ent + row);
          gb = -gh * 0.69314718055994530942;  // ln p = t ln 2
        }
        r.a = (float)(a * inv_t);
        r.b = (float)(gb * inv_t);
        r.xr = (float)((double)lse / inv_t);
        if (fabsf(lse) < CUDART_INF_F && fabsf(r.xr) < CUDART_INF_F) {
          r.k = (float)((((double)r.xr * inv_t - (double)lse) - tail) * kLog2eD);
          r.careful = fabsf(r.xr) >= 1e30f;
        } else {  // a row without a finite logit has no gradient
          r.xr = r.a = r.b = 0.f;
          r.k = -CUDART_INF_F;
          r.careful = 2;
        }
        sh_row = r;
      }
    }
    __syncthreads();
    const GradRow r = sh_row;
    const float xlow = r.xr - 200.0f / r.c2;
#pragma unroll
    for (int q = 0; q < kGradVecs; ++q) {
      const long long v = v0 + (q * kGradThreads + tid) * EV;
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
      } else if (v + EV > mis && v < end) {  // the vector that holds the row's first or last element
        for (int t = 0; t < EV; ++t) {
          const long long i = v + t - mis;
          if (i >= 0 && i < A.V) store_elem<DT>(outp, i, grad_one<ENT>(r, load_logit<DT>(rowp, i)));
        }
      }
    }
    __syncthreads();  // the chunk is written
    for (int e = tid; e < n_e; e += kGradThreads) {
      const int t = e_tok[e];
      const float x = e_x[e];
      if (!(fabsf(x) < CUDART_INF_F) || r.careful == 2) continue;
      const long long v = (long long)t + mis;
      if (v < v0 || v >= v0 + kChunk) continue;
      bool first = true;
      double g = 0.0;
      for (int o = 0; o < n_e; ++o) {
        if (e_tok[o] != t) continue;
        if (o < e) first = false;
        g += (double)e_g[o];
      }
      if (first) store_elem<DT>(outp, t, fmaf((float)g, r.inv_t, grad_one<ENT>(r, x)));
    }
    __syncthreads();  // the entries are free for the next chunk
  }
}

}  // namespace gls
