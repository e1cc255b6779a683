// gls_sample.cuh -- one token per row of logits by temperature, top-k, top-p and min-p, from a given uniform
// number.  With w_i = e^((l_i - max l) inv_temp) over the row's finite logits, in the order "larger logit
// first, ties by lower index", what is kept is always a start of the order:
//     top-k    the first k
//     top-p    the shortest start of those whose mass reaches p times theirs (rank r stays if the mass in front of
//              it is below p times the total)
//     min-p    the tokens with (l_i - max l) inv_temp >= ln(min_p)
// so it is described by the least kept logit and how many tokens of that logit stay (the lowest indices).
// The token is the first by INDEX whose cumulative kept mass exceeds u times the total.
//
// A CTA takes a row.  The row is read once from HBM; per chunk of 256 tokens (more in very long rows) the sweep
// keeps the largest logit and, where a total over the row is needed, the chunk's sum relative to it.  Everything
// later reads only the chunks whose largest logit reaches a bound, out of L2 (the rows in flight fit there):
//     bound    top-k: the k-th largest chunk maximum; top-p: V e^-c = (1 - p) total leaves no more than 1 - p
//              below max - c; min-p: itself
//     select   the least kept logit, by counting (and, for top-p, weighing) the tokens above the bound per bin of
//              their ordered codes and refining the bin the border falls into
//     sums     the kept tokens' mass per chunk, in 64 bits; the chunk that u falls into; the token inside it
// Decisions are those of exact arithmetic but for 64-bit rounding: sums that decide something are 64-bit sums of
// 64-bit exponentials (or integers of 2^-(62 - log2 V)).  The sweep's fp32 sums decide only where their error bound
// leaves no doubt; otherwise the row is summed again in 64 bits.
#pragma once
#include "gls_kernels.cuh"

namespace gls {

struct SampleSetting {
  const void* rows;       // NULL: `value` for every row
  long long sb, sk, sj;   // element strides
  float value;
  int ivalue;             // top_k
};

struct SampleArgs {
  const void* data;       // rows [B][K][J][V]
  long long sb, sk, sj;   // element strides
  int K, J, V;
  int shift;              // chunks of 256 << shift tokens
  SampleSetting inv_temp, top_k, top_p, min_p;
  const float* u;         // [B][K][J]
  int32_t* tokens;        // [B][K][J]
  float* logprobs;        // NULL or [B][K][J]
  uint32_t* status;
};

constexpr uint32_t kSampleBadSetting = 4u;  // GLS_DEV_BAD_SETTING
constexpr int kSampleBins = 2048;

__device__ __forceinline__ float redux_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
template <class T>
__device__ __forceinline__ T warp_scan(T x) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// A row in positions counted from the 16-byte boundary at or below its start: token i is position i + mis.
template <int DT>
struct SampleRow {
  static constexpr int ES = DT == kBF16 ? 2 : 4;
  static constexpr int kVec = ES / 2;  // 16-byte words per 8 positions
  struct Raw {
    uint4 v[kVec];
  };
  const char* base;
  long long mis, end;

  __device__ __forceinline__ Raw load(long long p) const {
    Raw r;
    if (p >= mis && p + 8 <= end) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) r.v[i] = __ldg((const uint4*)(base + p * ES) + i);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = p + i >= mis && p + i < end;
        if constexpr (DT == kBF16)
          w[i] = in ? (uint32_t)__ldg((const unsigned short*)base + p + i) : 0xff80u;
        else
          w[i] = in ? __ldg((const uint32_t*)base + p + i) : 0xff800000u;
      }
      if constexpr (DT == kBF16) {
        r.v[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
      } else {
        r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        r.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
    return r;
  }
  // masked logits (NaN, infinities) become -inf, -0 becomes +0
  static __device__ __forceinline__ void unpack(const Raw& r, float (&a)[8]) {
    if constexpr (DT == kBF16) {
      const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) a[2 * i] = bf16_lo(w[i]), a[2 * i + 1] = bf16_hi(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[4 * i] = __uint_as_float(r.v[i].x), a[4 * i + 1] = __uint_as_float(r.v[i].y);
        a[4 * i + 2] = __uint_as_float(r.v[i].z), a[4 * i + 3] = __uint_as_float(r.v[i].w);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = fabsf(a[i]) <= 3.402823466e38f ? a[i] + 0.f : -CUDART_INF_F;
  }
  // ordered code of a logit; bf16 logits have 16-bit codes, so that neighbouring codes are neighbouring values
  static __device__ __forceinline__ uint32_t key(float x) {
    const uint32_t e = enc_ordered(x);
    return DT == kBF16 ? e >> 16 : e;
  }
  static __device__ __forceinline__ float value(uint32_t k) {
    return dec_ordered(DT == kBF16 ? k << 16 | (k & 0x8000u ? 0u : 0xffffu) : k);
  }
  static constexpr uint32_t kLowest = DT == kBF16 ? 0x80u : 0x800000u;  // code of the lowest finite value
};

template <int THREADS>
struct SampleShared {
  static constexpr int kChunks = 2 * THREADS;
  double psum[kChunks];                     // mass per chunk
  unsigned long long mass[kSampleBins];     // per bin, in units of 2^-frac
  double wred[32];
  float cmax[kChunks], csum[kChunks];       // largest logit, sum relative to it
  uint32_t count[kSampleBins];
  uint32_t ired[32];
  uint16_t list[kChunks];                   // chunks to look at
  int n_list;
  // results of a search
  int found;
  uint32_t at;
  uint32_t nabove, nat;
  double mabove, mat;
  long long pos;
};

// exclusive prefix of x over the block; *total: the sum over all
template <int THREADS, class T>
__device__ __forceinline__ T block_scan(T x, T* red, T* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T incl = warp_scan(x);
  __syncthreads();  // earlier readers of red are done
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    const T y = red[w];
    if (w < warp) before += y;
    all += y;
  }
  *total = all;
  return before + (incl - x);
}

template <int DT, int THREADS>
struct Sampler {
  typedef SampleRow<DT> Row;
  typedef typename Row::Raw Raw;
  static constexpr int kWarps = THREADS / 32;
  static constexpr int kAhead = 4;
  static constexpr int kPer = kSampleBins / THREADS;  // bins per thread in a scan

  SampleShared<THREADS>& sh;
  Row row;
  int nch, shift, frac;
  double it;
  float top;  // the largest logit

  __device__ __forceinline__ double weight(float x) const { return exp(((double)x - (double)top) * it); }

  // f(chunk, first position of the lane, logits) over all chunks (LISTED: over sh.list), a warp per chunk
  template <bool LISTED, class Begin, class F, class End>
  __device__ __forceinline__ void for_chunks(Begin&& begin, F&& f, End&& fin) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = LISTED ? sh.n_list : nch;
    if (shift == 0) {
      for (int i0 = warp; i0 < n; i0 += kWarps * kAhead) {
        Raw r[kAhead];
        int c[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int i = i0 + q * kWarps;
          c[q] = i < n ? (LISTED ? (int)sh.list[i] : i) : -1;
          if (c[q] >= 0) r[q] = row.load((long long)c[q] * 256 + lane * 8);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          if (c[q] < 0) continue;
          float a[8];
          Row::unpack(r[q], a);
          begin(c[q]);
          f(c[q], (long long)c[q] * 256 + lane * 8, a);
          fin(c[q]);
        }
      }
      return;
    }
    for (int i = warp; i < n; i += kWarps) {
      const int c = LISTED ? (int)sh.list[i] : i;
      begin(c);
      for (long long p = ((long long)c << (8 + shift)) + lane * 8, e = (long long)(c + 1) << (8 + shift); p < e; p += 256) {
        float a[8];
        Row::unpack(row.load(p), a);
        f(c, p, a);
      }
      fin(c);
    }
  }

  // chunks whose largest logit reaches `bound` -> sh.list
  __device__ __forceinline__ void make_list(float bound) {
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    for (int c = threadIdx.x; c < nch; c += THREADS)
      if (sh.cmax[c] >= bound) sh.list[atomicAdd(&sh.n_list, 1)] = (uint16_t)c;
    __syncthreads();
  }

  // Largest logit (and, SUM, the sum of 2^((l - largest) c2)) of each chunk.
  template <bool SUM>
  __device__ __forceinline__ void sweep(float c2) {
    float m = 0.f, s = 0.f;
    for_chunks<false>([&](int) { m = -CUDART_INF_F, s = 0.f; },
                      [&](int, long long, const float (&a)[8]) {
                        const float mx = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(a[4], a[5]), fmaxf(a[6], a[7])));
                        const float nm = fmaxf(m, redux_max(mx));
                        if (SUM && nm > -CUDART_INF_F) {
                          float t = 0.f;
#pragma unroll
                          for (int i = 0; i < 8; ++i) t += ex2_approx((a[i] - nm) * c2);
                          s = s * (m > -CUDART_INF_F ? ex2_approx((m - nm) * c2) : 0.f) + t;
                        }
                        m = nm;
                      },
                      [&](int c) {
                        if (SUM) {
#pragma unroll
                          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                        }
                        if ((threadIdx.x & 31) == 0) {
                          sh.cmax[c] = m;
                          if (SUM) sh.csum[c] = s;
                        }
                      });
    __syncthreads();
  }

  // Tokens with codes in [lo, lo + span) per bin of 2^sh codes; MASS: their weights too.
  template <bool MASS>
  __device__ __forceinline__ void histogram(uint32_t lo, uint32_t span, int sft) {
    for (int i = threadIdx.x; i < kSampleBins; i += THREADS) {
      sh.count[i] = 0u;
      if (MASS) sh.mass[i] = 0ull;
    }
    __syncthreads();
    const double unit = (double)(1ull << frac);
    for_chunks<true>([](int) {},
                     [&](int, long long, const float (&a)[8]) {
#pragma unroll
                       for (int i = 0; i < 8; ++i) {
                         const uint32_t d = Row::key(a[i]) - lo;
                         if (d < span) {
                           atomicAdd(&sh.count[d >> sft], 1u);
                           if (MASS) atomicAdd(&sh.mass[d >> sft], (unsigned long long)(weight(a[i]) * unit + 0.5));
                         }
                       }
                     },
                     [](int) {});
    __syncthreads();
  }
  static __device__ __forceinline__ int bin_shift(uint32_t span) {
    const int bits = 32 - __clz((int)(span - 1u));
    return span <= 1u || bits <= 11 ? 0 : bits - 11;
  }

  // Code of the k-th largest chunk maximum (at least k tokens reach it); 0 where there are fewer chunks with one.
  __device__ uint32_t kth_chunk(uint32_t k) {
    constexpr int kEach = SampleShared<THREADS>::kChunks / 32;
    if (threadIdx.x < 32) {
      uint32_t code[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c = i * 32 + (int)threadIdx.x;
        code[i] = c < nch ? Row::key(sh.cmax[c]) : 0u;
      }
      uint32_t best = 0u;
      for (int bit = DT == kBF16 ? 15 : 31; bit >= 0; --bit) {
        const uint32_t cand = best | 1u << bit;
        uint32_t n = 0u;
#pragma unroll
        for (int i = 0; i < kEach; ++i) n += code[i] >= cand ? 1u : 0u;
        if (__reduce_add_sync(0xffffffffu, n) >= k) best = cand;
      }
      if (threadIdx.x == 0) sh.at = best;
    }
    __syncthreads();
    const uint32_t best = sh.at;
    __syncthreads();
    return best;
  }

  // The code of the k-th token of the order among codes >= lo, how many tokens of it stay, and how many have it;
  // false where fewer than k tokens are that large.
  __device__ bool kth(uint32_t lo, uint32_t k, uint32_t* code, uint32_t* take, uint32_t* equal) {
    uint32_t span = Row::key(top) - lo + 1u;
    for (;;) {
      const int sft = bin_shift(span);
      histogram<false>(lo, span, sft);
      uint32_t mine = 0u, total;
#pragma unroll
      for (int j = 0; j < kPer; ++j) mine += sh.count[kSampleBins - 1 - ((int)threadIdx.x * kPer + j)];
      uint32_t before = block_scan<THREADS>(mine, sh.ired, &total);
      if (total < k) return false;
      if (before < k && k <= before + mine) {
        for (int j = 0; j < kPer; ++j) {
          const int bin = kSampleBins - 1 - ((int)threadIdx.x * kPer + j);
          const uint32_t n = sh.count[bin];
          if (k <= before + n) {
            sh.at = (uint32_t)bin;
            sh.nabove = before;
            sh.nat = n;
            break;
          }
          before += n;
        }
      }
      __syncthreads();
      const uint32_t bin = sh.at;
      k -= sh.nabove;
      if (sft == 0) {
        *code = lo + bin;
        *take = k;
        *equal = sh.nat;
        __syncthreads();
        return true;
      }
      const uint32_t left = span - (bin << sft);
      lo += bin << sft;
      span = left < (1u << sft) ? left : 1u << sft;
      __syncthreads();
    }
  }

  // number of r in [0, n) with front + r w < goal
  static __device__ __forceinline__ uint32_t ranks_below(double front, double w, uint32_t n, double goal) {
    if (!(front < goal)) return 0u;
    const double q = (goal - front) / w;
    uint32_t r = q >= (double)n ? n : (uint32_t)q;
    while (r > 0u && !(front + (double)(r - 1u) * w < goal)) --r;
    while (r < n && front + (double)r * w < goal) ++r;
    return r;
  }

  // Least kept code under top-p among the codes >= lo (of those at lo, `drop` do not belong to the set).
  // Goal: share times the set's own mass, or somewhere between goal_lo and goal_hi.
  // 1: found; 0: the set does not reach the goal, all of it stays; -1: the interval leaves it open.
  __device__ int nucleus(uint32_t lo, uint32_t drop, bool own_total, double share, double goal_lo, double goal_hi,
                         uint32_t* code, uint32_t* take, uint32_t* equal) {
    uint32_t span = Row::key(top) - lo + 1u;
    const uint32_t first = lo;
    double above = 0.0;
    bool outermost = true;
    const double per_unit = 1.0 / (double)(1ull << frac);
    for (;;) {
      const int sft = bin_shift(span);
      if (sft == 0) histogram<false>(lo, span, sft);
      else histogram<true>(lo, span, sft);
      double m[kPer], mine = 0.0, total;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int bin = kSampleBins - 1 - ((int)threadIdx.x * kPer + j);
        uint32_t n = sh.count[bin];
        const bool lowest = bin == 0 && lo == first && drop > 0u;
        m[j] = 0.0;
        if (sft == 0) {
          if (lowest) n -= drop;
          if (n) m[j] = (double)n * weight(Row::value(lo + (uint32_t)bin));
        } else {
          if (n) m[j] = (double)sh.mass[bin] * per_unit;
          if (lowest) m[j] -= (double)drop * weight(Row::value(lo));
        }
        mine += m[j];
      }
      if (threadIdx.x == 0) sh.found = 0;
      double before = above + block_scan<THREADS>(mine, sh.wred, &total);
      if (own_total) {
        own_total = false;
        goal_lo = goal_hi = share * total;
      }
      const double goal = 0.5 * (goal_lo + goal_hi);
      if (before < goal && goal <= before + mine) {
        // the last bin that holds something where the bins' own sums round below the goal
        for (int j = 0; j < kPer; ++j) {
          if (m[j] > 0.0) {
            sh.found = 1;
            sh.at = (uint32_t)(kSampleBins - 1 - ((int)threadIdx.x * kPer + j));
            sh.mabove = before;
            if (goal <= before + m[j]) break;
          }
          before += m[j];
        }
      }
      __syncthreads();
      if (!sh.found) {
        __syncthreads();
        if (outermost) return above + total < goal_lo || goal_lo == goal_hi ? 0 : -1;
        // a bin whose parts' sum rounds below the bin's: its lowest part
        if (threadIdx.x == 0) {
          int bin = 0;
          while (bin < kSampleBins - 1 && sh.count[bin] == 0u) ++bin;
          sh.at = (uint32_t)bin;
          sh.mabove = above + total - (sft == 0 ? (double)sh.count[bin] * weight(Row::value(lo + (uint32_t)bin)) : (double)sh.mass[bin] * per_unit);
        }
        __syncthreads();
      }
      outermost = false;
      const uint32_t bin = sh.at;
      above = sh.mabove;
      if (sft == 0) {
        uint32_t n = sh.count[bin];
        *equal = n;
        if (lo + bin == first) n -= drop;
        *code = lo + bin;
        const double w = weight(Row::value(lo + bin));
        const uint32_t a = ranks_below(above, w, n, goal_lo), b = ranks_below(above, w, n, goal_hi);
        *take = b ? b : 1u;
        __syncthreads();
        if (goal_lo < goal_hi && (a != b || a == 0u || above + (double)n * w < goal_hi)) return -1;
        return 1;
      }
      const uint32_t left = span - (bin << sft);
      lo += bin << sft;
      span = left < (1u << sft) ? left : 1u << sft;
      __syncthreads();
    }
  }

  // Position behind the `take`-th token (by index) of this code; sh.list holds the chunks that may have some.
  __device__ long long equal_end(uint32_t code, uint32_t take) {
    uint32_t* cnt = (uint32_t*)sh.csum;  // the sweep's sums are not needed any more
    for (int c = threadIdx.x; c < SampleShared<THREADS>::kChunks; c += THREADS) cnt[c] = 0u;
    __syncthreads();
    uint32_t n = 0u;
    for_chunks<true>([&](int) { n = 0u; },
                     [&](int, long long, const float (&a)[8]) {
#pragma unroll
                       for (int i = 0; i < 8; ++i) n += Row::key(a[i]) == code ? 1u : 0u;
                     },
                     [&](int c) {
                       n = __reduce_add_sync(0xffffffffu, n);
                       if ((threadIdx.x & 31) == 0) cnt[c] = n;
                     });
    __syncthreads();
    const uint32_t x0 = cnt[2 * threadIdx.x], x1 = cnt[2 * threadIdx.x + 1];
    uint32_t total;
    const uint32_t before = block_scan<THREADS>(x0 + x1, sh.ired, &total);
    if (before < take && take <= before + x0) sh.at = 2 * threadIdx.x, sh.nabove = before;
    if (before + x0 < take && take <= before + x0 + x1) sh.at = 2 * threadIdx.x + 1, sh.nabove = before + x0;
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x, c = (int)sh.at;
      uint32_t want = take - sh.nabove;  // >= 1
      for (long long p0 = (long long)c << (8 + shift), e = (long long)(c + 1) << (8 + shift); p0 < e; p0 += 256) {
        float a[8];
        Row::unpack(row.load(p0 + lane * 8), a);
        uint32_t hits = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) hits |= (Row::key(a[i]) == code ? 1u : 0u) << i;
        const uint32_t mine = __popc(hits), incl = warp_scan(mine), all = __shfl_sync(0xffffffffu, incl, 31);
        if (want <= all) {
          if (incl - mine < want && want <= incl) {
            for (uint32_t r = incl - mine + 1u; r < want; ++r) hits &= hits - 1u;
            sh.pos = p0 + lane * 8 + __ffs((int)hits);
          }
          break;
        }
        want -= all;
      }
    }
    __syncthreads();
    const long long end = sh.pos;
    __syncthreads();
    return end;
  }

  struct Kept {
    uint32_t code;   // least kept code
    long long end;   // tokens of that code stay in front of this position
    __device__ __forceinline__ bool operator()(float x, long long p) const {
      const uint32_t k = Row::key(x);
      return k > code || (k == code && p < end);
    }
  };

  // 64-bit mass of the kept tokens of the listed chunks -> sh.psum, 0 elsewhere
  __device__ void exact_sums(const Kept& kept) {
    for (int c = threadIdx.x; c < SampleShared<THREADS>::kChunks; c += THREADS) sh.psum[c] = 0.0;
    __syncthreads();
    double s = 0.0;
    for_chunks<true>([&](int) { s = 0.0; },
                     [&](int, long long p, const float (&a)[8]) {
#pragma unroll
                       for (int i = 0; i < 8; ++i)
                         if (kept(a[i], p + i)) s += weight(a[i]);
                     },
                     [&](int c) {
                       s = warp_sum(s);
                       if ((threadIdx.x & 31) == 0) sh.psum[c] = s;
                     });
    __syncthreads();
  }
  __device__ double total_mass() {
    double total;
    block_scan<THREADS>(sh.psum[2 * threadIdx.x] + sh.psum[2 * threadIdx.x + 1], sh.wred, &total);
    return total;
  }

  // The token that u falls to by sh.psum.  slack: relative error of those sums; false where it leaves the token open.
  __device__ bool locate(const Kept& kept, double u, double slack, long long* pos, double* total_out) {
    const double x0 = sh.psum[2 * threadIdx.x], x1 = sh.psum[2 * threadIdx.x + 1];
    double total;
    const double before = block_scan<THREADS>(x0 + x1, sh.wred, &total);
    double x = u * total;
    const double most = total * (1.0 - 1.2e-16);
    if (x > most) x = most;
    if (threadIdx.x == 0) sh.found = 0, sh.pos = -1;
    __syncthreads();
    // the pieces' borders are rounded sums: where none holds x, the last chunk with mass does
    const bool in0 = x0 > 0.0 && before <= x && x < before + x0, in1 = x1 > 0.0 && before + x0 <= x && x < before + (x0 + x1);
    if (in0 || in1) {
      sh.at = 2 * threadIdx.x + (in0 ? 0 : 1);
      sh.mabove = in0 ? before : before + x0;
      sh.found = 1;
    }
    __syncthreads();
    if (!sh.found && threadIdx.x == 0) {
      double b = 0.0;
      for (int c = 0; c < nch; ++c)
        if (sh.psum[c] > 0.0 && (b <= x || !sh.found)) {
          sh.at = (uint32_t)c;
          sh.mabove = b;
          sh.found = 1;
          b += sh.psum[c];
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      const long long c = sh.at;
      double base = sh.mabove;
      const double margin = slack * total;
      long long last = -1;  // last kept position so far
      bool sure = true, done = false;
      for (long long p0 = c << (8 + shift), e = (c + 1) << (8 + shift); p0 < e && !done; p0 += 256) {
        const long long p = p0 + lane * 8;
        float a[8];
        Row::unpack(row.load(p), a);
        double w[8], mine = 0.0;
        int mlast = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = kept(a[i], p + i) ? weight(a[i]) : 0.0;
          mine += w[i];
          if (w[i] > 0.0) mlast = i;
        }
        const double incl = warp_scan(mine);
        const unsigned hit = __ballot_sync(0xffffffffu, base + incl > x && mine > 0.0);
        const unsigned some = __ballot_sync(0xffffffffu, mlast >= 0);
        if (hit) {
          const int src = __ffs((int)hit) - 1;
          if (lane == src) {
            double b = base + (incl - mine);
            int i = 0;
            // the lane's sums in order; the last of its kept tokens where rounding leaves none
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (w[j] > 0.0 && (i = j, b + w[j] > x)) break;
              else b += w[j];
            if (margin > 0.0) sure = x - b > margin && b + w[i] - x > margin;
            sh.pos = p + i;
            sh.found = sure ? 1 : 0;
          }
          done = true;
        } else if (some) {
          const int src = 31 - __clz((int)some);
          last = __shfl_sync(0xffffffffu, p + mlast, src);
        }
        base += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (!done && lane == 0) {
        sh.pos = last;
        sh.found = margin > 0.0 ? 0 : 1;
      }
    }
    __syncthreads();
    *pos = sh.pos;
    *total_out = total;
    const bool ok = sh.found != 0;
    __syncthreads();
    return ok && *pos >= 0;
  }
};

__device__ __forceinline__ float sample_setting(const SampleSetting& s, long long b, int k, int j) {
  return s.rows ? __ldg((const float*)s.rows + b * s.sb + k * s.sk + j * s.sj) : s.value;
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS) sample_kernel(const SampleArgs A) {
  typedef SampleRow<DT> Row;
  __shared__ SampleShared<THREADS> sh;
  Sampler<DT, THREADS> S{sh};
  const long long r = blockIdx.x;
  const int j = (int)(r % A.J), k = (int)(r / A.J % A.K);
  const long long b = r / A.J / A.K;
  float itf = sample_setting(A.inv_temp, b, k, j), p = sample_setting(A.top_p, b, k, j), mp = sample_setting(A.min_p, b, k, j);
  int kk = A.top_k.rows ? __ldg((const int*)A.top_k.rows + b * A.top_k.sb + k * A.top_k.sk + j * A.top_k.sj) : A.top_k.ivalue;
  const float u = __ldg(A.u + r);
  const bool greedy = itf == CUDART_INF_F;
  if (!((itf >= 1e-20f && itf <= 1e20f) || greedy) || !(p > 0.f) || !(mp >= 0.f && mp <= 1.f) || !(u >= 0.f && u <= 1.f)) {
    if (threadIdx.x == 0) {
      A.tokens[r] = -1;
      if (A.logprobs) A.logprobs[r] = 0.f;
      if (A.status) atomicOr(A.status, kSampleBadSetting);
    }
    return;
  }
  if (greedy) itf = 1.f, kk = 1;
  if (kk == 1) p = 1.f, mp = 0.f;
  const char* start = (const char*)A.data + (b * A.sb + k * A.sk + j * A.sj) * Row::ES;
  S.row.mis = ((uintptr_t)start & 15) / Row::ES;
  S.row.base = start - S.row.mis * Row::ES;
  S.row.end = S.row.mis + A.V;
  S.shift = A.shift;
  S.nch = (int)((S.row.end + (256LL << A.shift) - 1) >> (8 + A.shift));
  S.frac = 62 - (32 - __clz(A.V));
  S.it = (double)itf;
  const bool use_k = kk > 0 && kk < A.V, use_p = p < 1.f;
  const bool need_sum = !use_k && (use_p || mp == 0.f);
  const float c2 = itf * kLog2e;
  if (need_sum) S.template sweep<true>(c2);
  else S.template sweep<false>(c2);
  float m = -CUDART_INF_F;
  for (int c = threadIdx.x; c < S.nch; c += THREADS) m = fmaxf(m, sh.cmax[c]);
  m = redux_max(m);
  if ((threadIdx.x & 31) == 0) sh.ired[threadIdx.x >> 5] = __float_as_uint(m);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) m = fmaxf(m, __uint_as_float(sh.ired[w]));
  if (m == -CUDART_INF_F) {
    if (threadIdx.x == 0) {
      A.tokens[r] = -1;
      if (A.logprobs) A.logprobs[r] = 0.f;
      if (A.status) atomicOr(A.status, 1u);
    }
    return;
  }
  S.top = m;
  typename Sampler<DT, THREADS>::Kept kept{Row::kLowest, S.row.end};
  // Relative error of a chunk's sum: exponentials 2^-22; their arguments 3 roundings, weighted by the terms themselves
  // |t| is log2(chunk) + 1.5 on the mean; a chain of 2^shift + 13 additions.  One more step for what follows in 64 bits.
  const double eps = 2.5e-7 + 1.3e-7 * (9.5 + A.shift) + 6e-8 * (14.0 + (double)(1 << A.shift));
  double total = 0.0;
  long long pos = -1;
  bool done = false;
  if (need_sum) {
    for (int c = threadIdx.x; c < SampleShared<THREADS>::kChunks; c += THREADS)
      sh.psum[c] = c < S.nch && sh.cmax[c] > -CUDART_INF_F ? (double)sh.csum[c] * S.weight(sh.cmax[c]) : 0.0;
    __syncthreads();
    if (!use_p) done = S.locate(kept, (double)u, 2.2 * eps, &pos, &total);
  }
  if (!done) {
    // the least code that min-p keeps
    uint32_t floor_code = Row::kLowest;
    if (mp > 0.f) {
      const double ln = log((double)mp);
      float edge = (float)((double)m + ln / S.it);
      if (!(edge >= -3.402823466e38f)) edge = -3.402823466e38f;
      uint32_t e = Row::key(edge);
      const uint32_t hi = Row::key(m);
      if (e > hi) e = hi;
      while (e < hi && !(((double)Row::value(e) - (double)m) * S.it >= ln)) ++e;
      while (e > Row::kLowest && ((double)Row::value(e - 1) - (double)m) * S.it >= ln) --e;
      floor_code = e;
    }
    uint32_t take = 0u, equal = 0u;  // of the least kept code; equal == 0: all of it stays
    kept.code = floor_code;
    if (use_k) {
      // top-p needs the mass of all k
      uint32_t cut = use_p ? Row::kLowest : floor_code;
      if (kk <= S.nch) {
        const uint32_t e = S.kth_chunk((uint32_t)kk);
        if (e > cut) cut = e;
      }
      S.make_list(Row::value(cut));
      uint32_t code;
      const bool limited = S.kth(cut, (uint32_t)kk, &code, &take, &equal);
      if (limited) kept.code = code;
      else take = equal = 0u, kept.code = cut;
      if (limited && use_p) {
        uint32_t pc, pt, pe;
        const int got = S.nucleus(kept.code, equal - take, true, (double)p, 0.0, 0.0, &pc, &pt, &pe);
        if (got == 1) kept.code = pc, take = pt, equal = pe;
      }
      if (!limited && use_p) {  // fewer than k finite logits: all of them are the set
        uint32_t pc, pt, pe;
        const int got = S.nucleus(cut, 0u, true, (double)p, 0.0, 0.0, &pc, &pt, &pe);
        if (got == 1) kept.code = pc, take = pt, equal = pe;
      }
    } else if (use_p) {
      double goal = S.total_mass(), slack = eps;
      for (int pass = 0; pass < 2; ++pass) {
        // what lies below max - c has at most V e^(-c inv_temp) = (1 - p) total
        const double c = log((double)A.V / ((1.0 - (double)p) * goal * (1.0 - 2.0 * eps))) / S.it;
        float edge = (float)((double)m - (c > 0.0 ? c : 0.0) * (1.0 + 1e-6));
        if (!(edge >= -3.402823466e38f)) edge = -3.402823466e38f;
        uint32_t cut = Row::key(edge);
        if (cut > Row::kLowest) --cut;
        if (cut < floor_code) cut = floor_code;
        S.make_list(Row::value(cut));
        uint32_t pc, pt, pe;
        const int got = S.nucleus(cut, 0u, false, 0.0, (double)p * goal * (1.0 - slack), (double)p * goal * (1.0 + slack), &pc, &pt, &pe);
        if (got == 1) kept.code = pc, take = pt, equal = pe;
        else if (got == 0) kept.code = cut;
        if (got >= 0) break;
        // the border lies within the sweep's error: the total in 64 bits
        S.make_list(-3.402823466e38f);
        S.exact_sums(typename Sampler<DT, THREADS>::Kept{Row::kLowest, S.row.end});
        goal = S.total_mass();
        slack = 0.0;
      }
    }
    if (kept.code < floor_code) kept.code = floor_code, take = equal = 0u;
    S.make_list(Row::value(kept.code));
    kept.end = S.row.end;
    if (take < equal) kept.end = S.equal_end(kept.code, take);
    S.exact_sums(kept);
    S.locate(kept, (double)u, 0.0, &pos, &total);
  }
  if (threadIdx.x == 0) {
    if (pos < S.row.mis) pos = S.row.mis - 1;  // not reached: the largest logit is always kept
    A.tokens[r] = (int32_t)(pos - S.row.mis);
    if (A.logprobs && pos < S.row.mis) A.logprobs[r] = 0.f;
    else if (A.logprobs) {
      const float x = DT == kBF16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)S.row.base + pos) << 16)
                                  : __ldg((const float*)S.row.base + pos);
      A.logprobs[r] = (float)(((double)x - (double)m) * S.it - log(total));
    }
  }
}

}  // namespace gls
