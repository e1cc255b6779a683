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
// A CTA takes a row (a cluster of them sweeps it where there are few rows; the first one does the rest).  The row is read
// once from HBM; per chunk of 256 tokens (more in very long rows) the sweep keeps the largest logit and, where a total
// over the row is needed, per four chunks the sum relative to their largest.  Everything later reads only the chunks
// whose largest logit reaches a bound, out of L2 (the rows in flight fit there):
//     bound    top-k: the k-th largest chunk maximum; top-p: V e^-c = (1 - p) total leaves no more than 1 - p
//              below max - c; min-p: itself
//     select   the least kept logit, by counting (and, for top-p, weighing) the tokens above the bound per bin of
//              their ordered codes and refining the bin the border falls into
//     sums     the kept tokens' mass per chunk, in 64 bits; the chunk that u falls into; the token inside it
// Decisions are those of exact arithmetic but for 64-bit rounding: sums that decide something are 64-bit sums of
// exponentials good to 2e-13, and counts.  The sweep's fp32 sums decide only where the border is further away than they can be
// off at all (1.3e-6 of what they hold); otherwise the row is summed again in 64 bits.
#pragma once
#include "gls_async.cuh"
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

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_ctas() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// stores to the first CTA of the cluster
__device__ __forceinline__ void store_first(const float* at, float x) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(at), d;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(d) : "r"(a));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(d), "f"(x) : "memory");
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
  uint32_t mis, end;

  __device__ __forceinline__ Raw load(uint32_t p) const {
    Raw r;
    if (p >= mis && p + 8 <= end) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) r.v[i] = __ldg((const uint4*)(base + (long long)p * ES) + i);
    } else if (p >= end) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) r.v[i] = DT == kBF16 ? make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u)
                                                          : make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
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
  static __device__ __forceinline__ void widen(const Raw& r, float (&a)[8]) {
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
  }
  // the largest logit, +0 for -0; NaN counts as nothing (-inf)
  static __device__ __forceinline__ float largest(const Raw& r) {
    float m;
    if constexpr (DT == kBF16) {
      const uint32_t w = max_bf16x2(max_bf16x2(r.v[0].x, r.v[0].y), max_bf16x2(r.v[0].z, r.v[0].w));
      m = fmaxf(bf16_lo(w), bf16_hi(w));
    } else {
      float a[8];
      widen(r, a);
      m = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(a[4], a[5]), fmaxf(a[6], a[7])));
    }
    return fmaxf(m, -CUDART_INF_F) + 0.f;
  }
  // masked logits (NaN, infinities) become -inf, -0 becomes +0
  static __device__ __forceinline__ void unpack(const Raw& r, float (&a)[8]) {
    widen(r, a);
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

constexpr int kSampleChunks = 1024;
constexpr int kSampleList = 2048;

// Shared memory: what the search needs lies where the sweep's rings were.
template <int DT, int THREADS>
struct SampleShared {
  static constexpr int kStages = 2;
  static constexpr int kStage = DT == kBF16 ? 2048 : 4096;  // 1024 tokens
  union {
    struct {
      double psum[kSampleChunks];   // mass per chunk
      uint32_t count[kSampleBins];  // per bin, or per chunk
      uint32_t key[kSampleList], place[kSampleList];  // codes and positions of listed tokens, in order of position
    };
    char ring[THREADS / 32][kStages][kStage];
  };
  double wred[32];
  double exp16[16];             // 2^(i / 16)
  uint64_t barriers[THREADS / 32][kStages];
  float cmax[kSampleChunks];    // largest logit of a chunk
  float csum[kSampleChunks / 4];  // sum relative to the largest logit of four chunks
  uint32_t ired[32];
  uint16_t list[kSampleChunks];  // chunks to look at
  int n_list;
  // results of a search
  int found;
  uint32_t at;
  uint32_t nabove, nat;
  double mabove;
  uint32_t pos;
};

// the value of the lane in front, 0 in the first: from an inclusive scan what lies in front, with nothing taken off again (which
// would leave a small sum in front of a large term the rounding of the latter)
template <class T>
__device__ __forceinline__ T lane_before(T incl) {
  const T y = __shfl_up_sync(0xffffffffu, incl, 1);
  return threadIdx.x & 31 ? y : (T)0;
}
// Exclusive prefix of x over the block; *total: the sum over all; *end: where the next thread begins, to the bit.
template <int THREADS, class T>
__device__ __forceinline__ T block_scan(T x, T* red, T* total, T* end = nullptr) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T incl = warp_scan(x), front = lane_before(incl);
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
  if (end) *end = before + incl;
  return before + front;
}

template <int DT, int THREADS>
struct SampleCalls;

template <int DT, int THREADS>
struct Sampler {
  typedef SampleRow<DT> Row;
  typedef typename Row::Raw Raw;
  static constexpr int kWarps = THREADS / 32;
  static constexpr int kAhead = DT == kBF16 ? 4 : 2;
  static constexpr int kPer = kSampleBins / THREADS;     // bins per thread in a scan
  static constexpr int kPerC = kSampleChunks / THREADS;  // chunks

  typedef SampleShared<DT, THREADS> Shared;
  // (found anew in each function, so that the compiler sees that it is shared memory)
  static __device__ __forceinline__ Shared& shared() {
    extern __shared__ __align__(128) char sample_shared[];
    return *(Shared*)sample_shared;
  }
  Row row;
  int nch, shift;
  int listed;      // tokens in shared().key, or -1
  double it, it2;  // inverse temperature, the same to base 2
  double top64;    // the largest logit; exponent of a logit x: (x - top64) it2
  float top;       // the largest logit
  float least;     // below it weights are 0

  __device__ __forceinline__ void set_top(float m) {
    top = m;
    top64 = (double)m;
    // rounded up: at low temperatures a step of fp32 is many exponents, and weight_of's range ends at 2^-1022
    least = __double2float_ru(top64 - 1000.0 / it2);
  }
  // 2^((x - top) it2) to 2e-13 for x >= least: 2^n 2^(i / 16) 2^r with |r| <= 1 / 32, the last by its series (ten
  // operations in 64 bits and a conversion; exp() takes about three times as many).  The largest logit's is 1, so that sums and
  // shares of equal ones are exact.  Sixteen table entries have a pair of banks
  // each; with 64 a warp's reads wait for one another (7.8 a clock and SM).
  // (a number below 2^-1022 where it is not wanted, without a branch)
  __device__ __forceinline__ double weight_of(float x, bool wanted = true) const {
    const double d = (double)x - top64;
    const double magic = 6755399441055744.0 / 16.0;  // 1.5 * 2^48: sixteenths in the lowest bits
    const double big = fma(d, it2, magic);
    const int n = __double2loint(big);
    const double r = fma(d, it2, magic - big);
    double q = 1.3333558146428443e-3;  // ln2^5 / 5!
    q = fma(q, r, 9.6181291076284772e-3);
    q = fma(q, r, 5.5504108664821580e-2);
    q = fma(q, r, 2.4022650695910071e-1);
    q = fma(q, r, 6.9314718055994531e-1);
    const double e = shared().exp16[n & 15], y = fma(e * r, q, e);
    return __hiloint2double(wanted ? __double2hiint(y) + ((n >> 4) << 20) : 0, __double2loint(y));
  }
  __device__ __forceinline__ double weight(float x) const { return x >= least ? weight_of(x) : 0.0; }

  // f(chunk, first position of the lane, logits) over the chunks of sh.list, a warp per chunk; RAW: masked logits as they are
  template <bool RAW = false, class Begin, class F, class End>
  __device__ __forceinline__ void for_chunks(Begin&& begin, F&& f, End&& fin) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = shared().n_list;
    if (shift == 0) {
      // kAhead chunks of a warp at a time, the next ones requested before these are looked at
      Raw next[kAhead];
      auto fetch = [&](int i0) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int i = i0 + q * kWarps;
          if (i < n) next[q] = row.load((uint32_t)shared().list[i] * 256u + lane * 8);
        }
      };
      fetch(warp);
      for (int i0 = warp; i0 < n; i0 += kWarps * kAhead) {
        Raw r[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) r[q] = next[q];
        fetch(i0 + kWarps * kAhead);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int i = i0 + q * kWarps;
          if (i >= n) break;
          const int c = (int)shared().list[i];
          float a[8];
          if (RAW) Row::widen(r[q], a);
          else Row::unpack(r[q], a);
          begin(c);
          f(c, (uint32_t)c * 256u + lane * 8, a);
          fin(c);
        }
      }
      return;
    }
    for (int i = warp; i < n; i += kWarps) {
      const int c = (int)shared().list[i];
      begin(c);
      for (int i = 0; i < 1 << shift; ++i) {
        float a[8];
        const uint32_t p = ((uint32_t)c << (8 + shift)) + (uint32_t)i * 256u + lane * 8;
        if (RAW) Row::widen(row.load(p), a);
        else Row::unpack(row.load(p), a);
        f(c, p, a);
      }
      fin(c);
    }
  }

  // chunks whose largest logit reaches `bound` -> shared().list, in order
  __device__ __forceinline__ void make_list(float bound) {
    uint32_t in = 0u, total;
#pragma unroll
    for (int i = 0; i < kPerC; ++i) {
      const int c = (int)threadIdx.x * kPerC + i;
      if (c < nch && shared().cmax[c] >= bound) in |= 1u << i;
    }
    uint32_t at = block_scan<THREADS>((uint32_t)__popc(in), shared().ired, &total);
#pragma unroll
    for (int i = 0; i < kPerC; ++i)
      if (in >> i & 1u) shared().list[at++] = (uint16_t)(threadIdx.x * kPerC + i);
    if (threadIdx.x == 0) shared().n_list = (int)total;
    __syncthreads();
  }

  // The tokens with logits of `bound` and above -> shared().key and shared().place, in order of position; shared().list holds their chunks.
  // Sets `listed`; no more than there is room for, otherwise -1.
  __device__ __forceinline__ void gather(float bound, float upto) {
    uint32_t* const cnt = shared().count;  // per entry of the list
    uint32_t n = 0u;
    for (int i = threadIdx.x; i < kSampleChunks; i += THREADS) cnt[i] = 0u;
    __syncthreads();
    auto hits_of = [&](const float (&a)[8]) {
      uint32_t h = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) h |= (a[i] >= bound && a[i] <= upto ? 1u : 0u) << i;
      return h;
    };
    const int lane = threadIdx.x & 31;
    for_chunks<true>([&](int) { n = 0u; }, [&](int, uint32_t, const float (&a)[8]) { n += __popc(hits_of(a)); },
               [&](int c) {
                 n = __reduce_add_sync(0xffffffffu, n);
                 if (lane == 0) cnt[c] = n;
               });
    __syncthreads();
    uint32_t mine[kPerC], sum = 0u, total;
#pragma unroll
    for (int i = 0; i < kPerC; ++i) sum += mine[i] = cnt[threadIdx.x * kPerC + i];
    uint32_t at = block_scan<THREADS>(sum, shared().ired, &total);
    if (total > (uint32_t)kSampleList) {
      listed = -1;
      __syncthreads();
      return;
    }
#pragma unroll
    for (int i = 0; i < kPerC; ++i) {
      cnt[threadIdx.x * kPerC + i] = at;
      at += mine[i];
    }
    __syncthreads();
    for_chunks<true>([&](int c) { n = cnt[c]; },
               [&](int, uint32_t p, const float (&a)[8]) {
                 const uint32_t h = hits_of(a);
                 if (!__any_sync(0xffffffffu, h != 0u)) return;
                 const uint32_t k = __popc(h), incl = warp_scan(k);
                 uint32_t to = n + incl - k;
#pragma unroll
                 for (int i = 0; i < 8; ++i)
                   if (h >> i & 1u) {
                     shared().key[to] = Row::key(a[i] + 0.f);
                     shared().place[to++] = p + i;
                   }
                 n += __shfl_sync(0xffffffffu, incl, 31);
               },
               [](int) {});
    listed = (int)total;
    __syncthreads();
  }

  // Whether a set's sum is relative to ref, its largest logit times c2, rounded: the rounding stays in the exponents of all its
  // terms, half of one at most up to 2^24.  Beyond it (126 at 2^31: every term 0 or infinite) the largest logit is taken off
  // before the product.
  static __device__ __forceinline__ bool by_product(float ref) { return fabsf(ref) < 16777216.f; }

  // Largest logit of each chunk and, SUM, per four chunks the sum of 2^(l c2 - r) with r their largest one
  // times c2, rounded (where by_product does not hold: of 2^((l - their largest) c2)), into the shared memory
  // of the cluster's first CTA.  A warp takes every so many-th four chunks; those that lie within the row come
  // through a ring, two sets ahead.
  template <bool SUM>
  __device__ __forceinline__ void sweep(float c2) {
    constexpr int kStages = Shared::kStages;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)cluster_rank(), ranks = (int)cluster_ctas();
    const int sets = (nch + 3) >> 2, stride = kWarps * ranks, first = warp * ranks + rank;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(shared().ring[warp]), bars = (uint32_t)__cvta_generic_to_shared(shared().barriers[warp]);
    auto inside = [&](int g) { return shift == 0 && g * 1024LL >= row.mis && g * 1024LL + 1024 <= row.end; };
    auto request = [&](int g, int stage) {
      if (g < sets && inside(g) && elected()) {
        barrier_expect(bars + stage * 8, Shared::kStage);
        copy_bulk(ring + stage * Shared::kStage, row.base + (long long)g * Shared::kStage, Shared::kStage, bars + stage * 8);
      }
    };
    if (lane < kStages) barrier_init(bars + lane * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kStages; ++i) request(first + i * stride, i);
    uint32_t phases = 0u;
    int stage = 0;
    for (int g = first; g < sets; g += stride) {
      float m[4], s = 0.f;
      bool odd = true;  // to be looked at token by token
      if (inside(g)) {
        odd = !barrier_wait(bars + stage * 8, phases >> stage & 1u);
        phases ^= 1u << stage;
        __syncwarp();
        Raw r[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < Row::kVec; ++i)  // which lane has which token of a chunk does not matter here
            r[q].v[i] = *(const uint4*)(shared().ring[warp][stage] + (q * Row::kVec + i) * 512 + lane * 16);
        __syncwarp();
        request(g + kStages * stride, stage);
#pragma unroll
        for (int q = 0; q < 4; ++q) m[q] = redux_max(Row::largest(r[q]));
        const float mm = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        odd |= !(mm < CUDART_INF_F);
        const float ref = mm * c2;
        if (SUM && mm > -CUDART_INF_F) {
          odd |= !by_product(ref);
          float t[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float a[8];
            Row::widen(r[q], a);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = ex2_approx(fmaf(a[i], c2, -ref));
            t[q] = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
          }
          s = (t[0] + t[1]) + (t[2] + t[3]);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          odd |= !(s < CUDART_INF_F);  // a NaN among the logits
        }
      } else {
        request(g + kStages * stride, stage);
      }
      if (odd) {
        float4 q;
        s = SampleCalls<DT, THREADS>::sweep_carefully(*this, g, c2, SUM, &q);
        m[0] = q.x, m[1] = q.y, m[2] = q.z, m[3] = q.w;
      }
      if (lane < 4) {
        const float mine = lane == 0 ? m[0] : lane == 1 ? m[1] : lane == 2 ? m[2] : m[3];
        store_first(&shared().cmax[4 * g + lane], mine);
        if (SUM && lane == 0) store_first(&shared().csum[g], s);
      }
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }
  }
  // The same with masked logits taken out one by one, for chunks of any size.
  template <bool SUM>
  __device__ __forceinline__ float sweep_carefully(int g, float c2, float (&m)[4]) {
    const int lane = threadIdx.x & 31;
    float mm = -CUDART_INF_F;
    double s = 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      m[q] = -CUDART_INF_F;
      if (4 * g + q >= nch) continue;
      for (int k = 0; k < 1 << shift; ++k) {
        float a[8];
        Row::unpack(row.load(((uint32_t)(4 * g + q) << (8 + shift)) + (uint32_t)k * 256u + lane * 8), a);
        const float b = redux_max(fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(a[4], a[5]), fmaxf(a[6], a[7]))));
        m[q] = fmaxf(m[q], b);
        const float nm = fmaxf(mm, b);
        if (SUM && nm > -CUDART_INF_F) {
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] = ex2_approx((a[i] - nm) * c2);
          if (nm > mm) s *= mm > -CUDART_INF_F ? exp2(((double)mm - (double)nm) * (double)c2) : 0.0;
          s += (double)(((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7])));
        }
        mm = nm;
      }
    }
    if (SUM) s = warp_sum(s);
    if (SUM && by_product(mm * c2)) s *= exp2((double)mm * (double)c2 - (double)(mm * c2));  // to the reference that sets without odd logits have
    return (float)s;
  }

  // Tokens with codes in [lo, lo + span) per bin of 2^sft codes, of the listed tokens or of the listed chunks.  (32-bit
  // counts: 12 a clock and SM; 64-bit sums of weights would be 1.6, and 0.35 where a few bins take them.)
  __device__ __forceinline__ void histogram(uint32_t lo, uint32_t span, int sft) {
    for (int i = threadIdx.x; i < kSampleBins; i += THREADS) shared().count[i] = 0u;
    __syncthreads();
    if (listed >= 0) {
      for (int i = threadIdx.x; i < listed; i += THREADS) {
        const uint32_t d = shared().key[i] - lo;
        if (d < span) atomicAdd(&shared().count[d >> sft], 1u);
      }
    } else {
      const float from = Row::value(lo), upto = top;
      for_chunks<true>([](int) {},
                 [&](int, uint32_t, const float (&a)[8]) {
#pragma unroll
                   for (int i = 0; i < 8; ++i)
                     if (a[i] >= from && a[i] <= upto) {
                       const uint32_t d = Row::key(a[i] + 0.f) - lo;
                       if (d < span) atomicAdd(&shared().count[d >> sft], 1u);
                     }
                 },
                 [](int) {});
    }
    __syncthreads();
  }
  // 64-bit mass of the tokens with codes lo .. hi
  __device__ __forceinline__ double mass_of(uint32_t lo, uint32_t hi) {
    if (listed < 0) {
      exact_sums(Kept{Row::value(lo), Row::value(hi), row.end});
      return total_mass();
    }
    double mine = 0.0, total;
    for (int i = threadIdx.x; i < listed; i += THREADS) {
      const uint32_t k = shared().key[i];
      if (k >= lo && k <= hi) mine += weight(Row::value(k));
    }
    block_scan<THREADS>(mine, shared().wred, &total);
    return total;
  }
  static __device__ __forceinline__ int bin_shift(uint32_t span) {
    const int bits = 32 - __clz((int)(span - 1u));
    return span <= 1u || bits <= 11 ? 0 : bits - 11;
  }

  // Code of the k-th largest chunk maximum (at least k tokens reach it); 0 where there are fewer chunks with one.
  __device__ __forceinline__ uint32_t kth_chunk(uint32_t k) {
    constexpr int kEach = kSampleChunks / 32;
    if (threadIdx.x < 32) {
      uint32_t code[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c = i * 32 + (int)threadIdx.x;
        code[i] = c < nch ? Row::key(shared().cmax[c]) : 0u;
      }
      uint32_t best = 0u;
      for (int bit = DT == kBF16 ? 15 : 31; bit >= 0; --bit) {
        const uint32_t cand = best | 1u << bit;
        uint32_t n = 0u;
#pragma unroll
        for (int i = 0; i < kEach; ++i) n += code[i] >= cand ? 1u : 0u;
        if (__reduce_add_sync(0xffffffffu, n) >= k) best = cand;
      }
      if (threadIdx.x == 0) shared().at = best;
    }
    __syncthreads();
    const uint32_t best = shared().at;
    __syncthreads();
    return best;
  }

  // The code of the k-th token of the order among codes >= lo, how many tokens of it stay, and how many have it;
  // false where fewer than k tokens are that large.
  __device__ __forceinline__ bool kth(uint32_t lo, uint32_t k, uint32_t* code, uint32_t* take, uint32_t* equal) {
    uint32_t span = Row::key(top) - lo + 1u;
    for (;;) {
      const int sft = bin_shift(span);
      histogram(lo, span, sft);
      uint32_t mine = 0u, total;
#pragma unroll
      for (int j = 0; j < kPer; ++j) mine += shared().count[kSampleBins - 1 - ((int)threadIdx.x * kPer + j)];
      uint32_t before = block_scan<THREADS>(mine, shared().ired, &total);
      if (total < k) return false;
      if (before < k && k <= before + mine) {
        for (int j = 0; j < kPer; ++j) {
          const int bin = kSampleBins - 1 - ((int)threadIdx.x * kPer + j);
          const uint32_t n = shared().count[bin];
          if (k <= before + n) {
            shared().at = (uint32_t)bin;
            shared().nabove = before;
            shared().nat = n;
            break;
          }
          before += n;
        }
      }
      __syncthreads();
      const uint32_t bin = shared().at;
      k -= shared().nabove;
      if (sft == 0) {
        *code = lo + bin;
        *take = k;
        *equal = shared().nat;
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
    // off by its rounding; by more than one where many such weights are less than a step of the sum: by halving
    if ((r == 0u || front + (double)(r - 1u) * w < goal) && (r == n || !(front + (double)r * w < goal))) return r;
    uint32_t lo = 0u, hi = n;
    while (lo < hi) {
      const uint32_t c = lo + (hi - lo) / 2u;
      if (front + (double)c * w < goal) lo = c + 1u;
      else hi = c;
    }
    return lo;
  }

  // Least kept code under top-p among the codes >= lo (of those at lo, `drop` do not belong to the set).
  // Goal: share times the set's own mass, or somewhere between goal_lo and goal_hi.  counted: the bins hold the counts of a call
  // with the same lo, whose codes had a bin each.
  // 1: found; 0: the set does not reach the goal, all of it stays; -1: the interval leaves it open.
  // Bins of one code have their mass from their count.  The masses of wider ones lie between their counts times the
  // weights at their ends, which leaves a few bins that the border may be in: the mass above those is summed in 64 bits
  // and they are cut finer, among their own tokens only as soon as there is room for these.
  __device__ __forceinline__ int nucleus(uint32_t lo, uint32_t drop, bool own_total, bool counted, double share, double goal_lo, double goal_hi,
                                         uint32_t* code, uint32_t* take, uint32_t* equal) {
    const uint32_t first = lo;
    uint32_t hi = Row::key(top);
    double above = 0.0;  // mass of the codes above hi
    if (own_total) goal_lo = goal_hi = share * (mass_of(lo, hi) - (double)drop * weight(Row::value(lo)));
    const double goal = 0.5 * (goal_lo + goal_hi);
    for (;;) {
      const uint32_t span = hi - lo + 1u;
      const int sft = bin_shift(span);
      if (!counted) histogram(lo, span, sft);
      counted = false;
      if (lo == first && drop > 0u) {
        if (threadIdx.x == 0) shared().count[0] -= drop;
        __syncthreads();
      }
      // masses from the top bin on: at least and at most
      double least_sum = 0.0, most_sum = 0.0, total_least, total_most;
#pragma unroll 1
      for (int j = 0; j < kPer; ++j) {
        const uint32_t bin = kSampleBins - 1 - (threadIdx.x * kPer + j), n = shared().count[bin];
        if (!n) continue;
        const uint32_t c0 = lo + (bin << sft), c1 = min(c0 + (1u << sft) - 1u, hi);
        const double w = (double)n * weight(Row::value(c1));
        most_sum += w;
        least_sum += sft == 0 ? w : (double)n * weight(Row::value(c0));
      }
      if (threadIdx.x == 0) shared().found = 0, shared().at = 0xffffffffu, shared().nat = 0u;
      const double most0 = above + block_scan<THREADS>(most_sum, shared().wred, &total_most);
      if (sft == 0) {
        if (most0 < goal && goal <= most0 + most_sum) {
          double before = most0;
          // the last bin that holds something where the bins' own sums round below the goal
          for (int j = 0; j < kPer; ++j) {
            const uint32_t bin = kSampleBins - 1 - (threadIdx.x * kPer + j), n = shared().count[bin];
            if (!n) continue;
            const double w = (double)n * weight(Row::value(lo + bin));
            shared().found = 1;
            shared().at = bin;
            shared().mabove = before;
            before += w;
            if (goal <= before) break;
          }
        }
        __syncthreads();
        if (!shared().found) {
          const bool whole = lo == first;
          if (whole) {
            __syncthreads();
            return above + total_most < goal_lo || goal_lo == goal_hi ? 0 : -1;
          }
          // a border that rounding put behind the last code of the bins it was found in
          if (threadIdx.x == 0) {
            uint32_t bin = 0u;
            while (bin < kSampleBins - 1 && shared().count[bin] == 0u) ++bin;
            shared().at = bin;
            shared().mabove = above + total_most - (double)shared().count[bin] * weight(Row::value(lo + bin));
          }
          __syncthreads();
        }
        const uint32_t bin = shared().at, n = shared().count[bin];
        above = shared().mabove;
        *code = lo + bin;
        *equal = n + (lo + bin == first ? drop : 0u);
        const double w = weight(Row::value(lo + bin));
        const uint32_t a = ranks_below(above, w, n, goal_lo), b = ranks_below(above, w, n, goal_hi);
        *take = b ? b : 1u;
        __syncthreads();
        if (goal_lo < goal_hi && (a != b || a == 0u || above + (double)n * w < goal_hi)) return -1;
        return 1;
      }
      const double least0 = above + block_scan<THREADS>(least_sum, shared().wred, &total_least);
      // The border lies no higher than the first bin with which the masses at most reach the goal, and no lower than the first
      // with which those at least do (2^-40 of the goal wider, for the sums' own rounding).
      const double from = goal_lo * (1.0 - 1e-12), upto = goal_hi * (1.0 + 1e-12);
      const bool top_here = most0 < from && from <= most0 + most_sum, low_here = least0 < upto && upto <= least0 + least_sum;
      if (top_here || low_here) {
        double f = most0, g = least0;
        bool top_open = top_here, low_open = low_here;
        for (int j = 0; j < kPer; ++j) {
          const uint32_t bin = kSampleBins - 1 - (threadIdx.x * kPer + j), n = shared().count[bin];
          if (!n) continue;
          const uint32_t c0 = lo + (bin << sft), c1 = min(c0 + (1u << sft) - 1u, hi);
          if (top_open) {
            shared().at = bin;
            f += (double)n * weight(Row::value(c1));
            top_open = f < from;
          }
          if (low_open) {
            shared().nat = bin;
            g += (double)n * weight(Row::value(c0));
            low_open = g < upto;
          }
        }
      }
      __syncthreads();
      const uint32_t b1 = shared().at, b0 = shared().nat;
      __syncthreads();
      if (b1 == 0xffffffffu) {
        if (lo == first) return above + total_most < goal_lo ? 0 : goal_lo == goal_hi ? 0 : -1;
        // rounding again: the lowest bin that holds something
        if (threadIdx.x == 0) {
          uint32_t bin = 0u;
          while (bin < kSampleBins - 1 && shared().count[bin] == 0u) ++bin;
          shared().at = bin;
        }
        __syncthreads();
      }
      const uint32_t bin1 = shared().at, upper = min(lo + (bin1 << sft) + ((1u << sft) - 1u), hi);
      uint32_t lower = lo + (b0 << sft), edge = upper;
      __syncthreads();
      if (upper == hi && lower == lo) {
        // bins too wide for their ends to say anything: whether the border is in the first of them decides its mass
        const uint32_t low1 = lo + (bin1 << sft);
        const double in_it = mass_of(low1, hi);
        if (above + in_it >= goal) {
          lower = low1;  // above lo: a bin is narrower than the span
        } else {
          above += in_it;
          edge = low1 - 1u;
          hi = edge;
          continue;
        }
      } else if (upper < hi) {
        above += mass_of(upper + 1u, hi);
      }
      // few tokens left: they alone are looked at from here on
      if (listed < 0) {
        uint32_t mine = 0u, left;
#pragma unroll 1
        for (int j = 0; j < kPer; ++j) {
          const uint32_t bin = kSampleBins - 1 - (threadIdx.x * kPer + j);
          if (bin >= b0 && bin <= bin1) mine += shared().count[bin];
        }
        block_scan<THREADS>(mine, shared().ired, &left);
        if (left <= (uint32_t)kSampleList) listed = SampleCalls<DT, THREADS>::gather(*this, Row::value(max(lower, first)), Row::value(edge));
      }
      hi = edge;
      if (lower > hi) lower = hi;
      lo = lower;
    }
  }

  // Position behind the `take`-th token (by index) of this code; shared().list holds the chunks that may have some.
  __device__ __forceinline__ uint32_t equal_end(uint32_t code, uint32_t take) {
    uint32_t* cnt = shared().count;
    for (int c = threadIdx.x; c < kSampleChunks; c += THREADS) cnt[c] = 0u;
    __syncthreads();
    uint32_t n = 0u;
    const float value = Row::value(code);
    for_chunks<true>([&](int) { n = 0u; },
               [&](int, uint32_t, const float (&a)[8]) {
#pragma unroll
                 for (int i = 0; i < 8; ++i) n += a[i] == value ? 1u : 0u;
               },
               [&](int c) {
                 n = __reduce_add_sync(0xffffffffu, n);
                 if ((threadIdx.x & 31) == 0) cnt[c] = n;
               });
    __syncthreads();
    uint32_t mine = 0u, total;
#pragma unroll
    for (int i = 0; i < kPerC; ++i) mine += cnt[threadIdx.x * kPerC + i];
    uint32_t before = block_scan<THREADS>(mine, shared().ired, &total);
    if (before < take && take <= before + mine) {
      for (int i = 0; i < kPerC; ++i) {
        const uint32_t x = cnt[threadIdx.x * kPerC + i];
        if (take <= before + x) {
          shared().at = threadIdx.x * kPerC + i;
          shared().nabove = before;
          break;
        }
        before += x;
      }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x, c = (int)shared().at;
      uint32_t want = take - shared().nabove;  // >= 1
      for (int k = 0; k < 1 << shift; ++k) {
        const uint32_t p0 = ((uint32_t)c << (8 + shift)) + (uint32_t)k * 256u;
        float a[8];
        Row::unpack(row.load(p0 + lane * 8), a);
        uint32_t hits = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) hits |= (Row::key(a[i]) == code ? 1u : 0u) << i;
        const uint32_t mine = __popc(hits), incl = warp_scan(mine), all = __shfl_sync(0xffffffffu, incl, 31);
        if (want <= all) {
          if (incl - mine < want && want <= incl) {
            for (uint32_t r = incl - mine + 1u; r < want; ++r) hits &= hits - 1u;
            shared().pos = p0 + lane * 8 + __ffs((int)hits);
          }
          break;
        }
        want -= all;
      }
    }
    __syncthreads();
    const uint32_t end = shared().pos;
    __syncthreads();
    return end;
  }

  struct Kept {
    float from;    // least kept logit
    float upto;    // the largest one (+inf and NaN are not kept)
    uint32_t end;  // tokens of the least one stay in front of this position
    __device__ __forceinline__ bool operator()(float x, uint32_t p) const {
      return x >= from && x <= upto && !(x == from && p >= end);
    }
  };

  // The kept ones' mass among a lane's eight tokens, without branches, since a weight's operations wait for one another;
  // not computed where no lane has a kept one.
  __device__ __forceinline__ double kept_mass(const Kept& kept, const float (&a)[8], uint32_t p) const {
    const float from = fmaxf(kept.from, least);
    bool keep[8], any = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      bool in = a[i] >= from && a[i] <= kept.upto;
      if (p + 8u > kept.end) in = in && !(p + i >= kept.end && a[i] == kept.from);  // some of the least ones are out
      any |= keep[i] = in;
    }
    if (!__any_sync(0xffffffffu, any)) return 0.0;
    double s = 0.0;
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      double w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = weight_of(a[h + i], keep[h + i]);
      s += (w[0] + w[1]) + (w[2] + w[3]);
    }
    return s;
  }

  // 64-bit mass of the kept tokens of the listed chunks -> shared().psum, 0 elsewhere
  __device__ __forceinline__ void exact_sums(const Kept& kept) {
    for (int c = threadIdx.x; c < kSampleChunks; c += THREADS) shared().psum[c] = 0.0;
    __syncthreads();
    double s = 0.0;
    for_chunks<true>([&](int) { s = 0.0; },
                     [&](int, uint32_t p, const float (&a)[8]) {
                       s += kept_mass(kept, a, p);
                     },
                     [&](int c) {
                       s = warp_sum(s);
                       if ((threadIdx.x & 31) == 0) shared().psum[c] = s;
                     });
    __syncthreads();
  }
  __device__ double total_mass() {
    double mine = 0.0, total;
#pragma unroll
    for (int i = 0; i < kPerC; ++i) mine += shared().psum[threadIdx.x * kPerC + i];
    block_scan<THREADS>(mine, shared().wred, &total);
    return total;
  }

  // The token that u falls to by shared().psum, whose entries hold 2^size positions each.  slack: relative error of those sums;
  // false where it leaves the token open, or where there is no mass.  The entry that u falls into is looked at in 64 bits.
  // With sums S = M (1 + e) and P in front of that entry, u total - P is off by u times the errors from the entry on minus (1 - u)
  // times those in front of it: by slack ((1 - u) P + u (total - P)) at most.
  __device__ __forceinline__ bool locate(const Kept& kept, double u, int size, double slack, uint32_t* pos, double* total_out) {
    double mine = 0.0, total, end;
#pragma unroll
    for (int i = 0; i < kPerC; ++i) mine += shared().psum[threadIdx.x * kPerC + i];
    if (threadIdx.x == 0) shared().at = 0u, shared().mabove = 0.0;
    double before = block_scan<THREADS>(mine, shared().wred, &total, &end);
    if (!(total > 0.0 && total < CUDART_INF)) return false;  // no entry to look into
    double x = u * total;
    const double most = total * (1.0 - 1.2e-16);
    if (x > most) x = most;
        if (before <= x && x < end) {
      for (int i = 0; i < kPerC; ++i) {
        const double y = shared().psum[threadIdx.x * kPerC + i];
        if (y > 0.0) {
          shared().at = threadIdx.x * kPerC + i;
          shared().mabove = before;
          if (x < before + y) break;
        }
        before += y;
      }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      const double first = shared().mabove;
      const double margin = slack > 0.0 ? slack * ((1.0 - u) * first + u * (total - first)) + 1e-12 * total : 0.0;
      double front = first;
      uint32_t last = row.mis;  // last kept position so far
      bool sure = true, done = false, likely = false;
      const int parts = 1 << (size - 8);
      for (int k = 0; k < parts && (!done || likely); ++k) {
        const uint32_t p = (shared().at << size) + (uint32_t)k * 256u + lane * 8;
        float a[8];
        Row::unpack(row.load(p), a);
        double w[8], mine = 0.0;
        int mlast = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = weight(a[i]);
          if (!kept(a[i], p + i)) w[i] = 0.0;
          mine += w[i];
          if (w[i] > 0.0) mlast = i;
        }
        const double incl = warp_scan(mine), ahead = lane_before(incl);
        const unsigned hit = __ballot_sync(0xffffffffu, front + incl > x && mine > 0.0);
        const unsigned some = __ballot_sync(0xffffffffu, mlast >= 0);
        if (!done && hit) {
          const int src = __ffs((int)hit) - 1;
          bool half = false;
          if (lane == src) {
            double f = front + ahead, border = f;
            int at = 0;
            bool open = true;
            // the lane's sums in order; the last of its kept tokens where rounding leaves none
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (open && w[i] > 0.0) {
                at = i;
                border = f;
                f += w[i];
                open = !(f > x);
              }
            if (margin > 0.0) sure = x - border > margin && f - x > margin;
            shared().pos = p + at;
            shared().found = sure ? 1 : 0;
            half = slack > 0.0 && f - border > 0.5 * total;
          }
          done = true;
          likely = __any_sync(0xffffffffu, half);
        } else if (some) {
          const int src = 31 - __clz((int)some);
          last = __shfl_sync(0xffffffffu, p + mlast, src);
        }
        front += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (!done && lane == 0) {
        shared().pos = last;
        shared().found = slack > 0.0 ? 0 : 1;
      }
      // for a token that has more than half of it the total has the entry's own mass in 64 bits: its log probability is near 0, and off
      // by a share of what others hold
      if (lane == 0) shared().mabove = likely ? total - shared().psum[shared().at] + (front - first) : total;
    }
    __syncthreads();
    *total_out = shared().mabove;
    *pos = shared().pos;
    const bool ok = shared().found != 0;
    __syncthreads();
    return ok;
  }

  // All of it for no more listed tokens than threads, which are at least the first `k` of the order or all of it: a thread has
  // one, finds its place in the order by comparing it with the others, and top-p's border and the token that u falls to
  // are scans over the threads.
  __device__ __forceinline__ void pick(uint32_t k, bool use_p, double share, uint32_t floor_code, double u, uint32_t* pos, double* total_out) {
    const int i = threadIdx.x;
    const bool have = i < listed;
    const uint32_t mine = have ? shared().key[i] : 0u;
    uint32_t rank = 0u;
    for (int j = 0; j < listed; ++j) {
      const uint32_t other = shared().key[j];
      rank += other > mine || (other == mine && j < i) ? 1u : 0u;
    }
    const double w = have ? weight(Row::value(mine)) : 0.0;
    double total;
    if (use_p) {
      shared().psum[i] = 0.0;
      __syncthreads();
      if (have && rank < k) shared().psum[rank] = w;
      __syncthreads();
      const double x = shared().psum[i], front = block_scan<THREADS>(x, shared().wred, &total);
      const uint32_t stay = (uint32_t)__syncthreads_count((uint32_t)i < k && i < listed && front < share * total);
      if (stay < k) k = stay ? stay : 1u;
    }
    const bool kept = have && (rank < k && mine >= floor_code || rank == 0u);
    double end;
    const double y = kept ? w : 0.0, f = block_scan<THREADS>(y, shared().wred, &total, &end);
    double x = u * total;
    const double most = total * (1.0 - 1.2e-16);
    if (x > most) x = most;
    if (i == 0) shared().found = 0, shared().at = u == 0.0 ? 0xffffffffu : 0u;
    __syncthreads();
    if (y > 0.0) {
      // for u = 1 the last one with weight, for u = 0 the first
      if (u == 0.0) atomicMin(&shared().at, (uint32_t)i);
      else atomicMax(&shared().at, (uint32_t)i);
      if (u > 0.0 && u < 1.0 && f <= x && x < end) {
        shared().pos = shared().place[i];
        shared().found = 1;
      }
    }
    __syncthreads();
    *pos = shared().found ? shared().pos : shared().place[shared().at];
    *total_out = total;
  }

  // The same among the listed tokens, of which the first `take` (by position) of the code `code` and those above it stay.
  __device__ __forceinline__ void locate_listed(uint32_t code, uint32_t take, double u, uint32_t* pos, double* total_out) {
    const int each = (listed + THREADS - 1) / THREADS, from = min((int)threadIdx.x * each, listed), upto = min(from + each, listed);
    uint32_t equal = 0u, all;
    for (int i = from; i < upto; ++i) equal += shared().key[i] == code ? 1u : 0u;
    const uint32_t rank = block_scan<THREADS>(equal, shared().ired, &all);
    double mine = 0.0, total, end;
    uint32_t r = rank;
    for (int i = from; i < upto; ++i) {
      const uint32_t k = shared().key[i];
      if (k > code || (k == code && r++ < take)) mine += weight(Row::value(k));
    }
    if (threadIdx.x == 0) shared().pos = row.mis;
    double f = block_scan<THREADS>(mine, shared().wred, &total, &end);
    double x = u * total;
    const double most = total * (1.0 - 1.2e-16);
    if (x > most) x = most;
    if (u > 0.0 && u < 1.0 && f <= x && x < end) {
      r = rank;
      for (int i = from; i < upto; ++i) {
        const uint32_t k = shared().key[i];
        if (!(k > code || (k == code && r++ < take))) continue;
        const double w = weight(Row::value(k));
        if (!(w > 0.0)) continue;
        shared().pos = shared().place[i];
        f += w;
        if (f > x) break;
      }
    }
    __syncthreads();
    // for u = 1 the last token with weight, for u = 0 the first
    if (!(u > 0.0 && u < 1.0) && threadIdx.x == 0) {
      r = 0u;
      for (int i = 0; i < listed; ++i) {
        const uint32_t k = shared().key[i];
        if (!(k > code || (k == code && r++ < take)) || !(weight(Row::value(k)) > 0.0)) continue;
        shared().pos = shared().place[i];
        if (u == 0.0) break;
      }
    }
    __syncthreads();
    *pos = shared().pos;
    *total_out = total;
    __syncthreads();
  }
};

// The searches as functions of their own (inlined, the kernel would not fit its registers), each with a copy of the
// sampler that it can hold in registers.
template <int DT, int THREADS>
struct SampleCalls {
  typedef Sampler<DT, THREADS> S;
  typedef typename S::Kept Kept;
  static __device__ __noinline__ float sweep_carefully(S s, int g, float c2, bool sum, float4* m) {
    float q[4];
    const float t = sum ? s.template sweep_carefully<true>(g, c2, q) : s.template sweep_carefully<false>(g, c2, q);
    *m = make_float4(q[0], q[1], q[2], q[3]);
    return t;
  }
  static __device__ __noinline__ uint32_t kth_chunk(S s, uint32_t k) { return s.kth_chunk(k); }
  static __device__ __noinline__ void make_list(S s, float bound) { s.make_list(bound); }
  static __device__ __noinline__ int gather(S s, float bound, float upto) {
    s.gather(bound, upto);
    return s.listed;
  }
  static __device__ __noinline__ bool kth(S s, uint32_t lo, uint32_t k, uint32_t* code, uint32_t* take, uint32_t* equal) {
    return s.kth(lo, k, code, take, equal);
  }
  static __device__ __noinline__ int nucleus(S s, uint32_t lo, uint32_t drop, bool own, bool counted, double share, double goal_lo, double goal_hi,
                                             uint32_t* code, uint32_t* take, uint32_t* equal) {
    return s.nucleus(lo, drop, own, counted, share, goal_lo, goal_hi, code, take, equal);
  }
  static __device__ __noinline__ uint32_t equal_end(S s, uint32_t code, uint32_t take) { return s.equal_end(code, take); }
  static __device__ __noinline__ void exact_sums(S s, Kept kept) { s.exact_sums(kept); }
  static __device__ __noinline__ bool locate(S s, Kept kept, double u, int size, double slack, uint32_t* pos, double* total) {
    return s.locate(kept, u, size, slack, pos, total);
  }
  static __device__ __noinline__ void pick(S s, uint32_t k, bool use_p, double share, uint32_t floor_code, double u, uint32_t* pos,
                                           double* total) {
    s.pick(k, use_p, share, floor_code, u, pos, total);
  }
  static __device__ __noinline__ void locate_listed(S s, uint32_t code, uint32_t take, double u, uint32_t* pos, double* total) {
    s.locate_listed(code, take, u, pos, total);
  }
};

__device__ __forceinline__ float sample_setting(const SampleSetting& s, long long b, int k, int j) {
  return s.rows ? __ldg((const float*)s.rows + b * s.sb + k * s.sk + j * s.sj) : s.value;
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 1 : 1024 / THREADS) sample_kernel(const SampleArgs A) {
  typedef SampleRow<DT> Row;
  typedef SampleCalls<DT, THREADS> Calls;
  SampleShared<DT, THREADS>& sh = Sampler<DT, THREADS>::shared();
  Sampler<DT, THREADS> S;
  const long long r = blockIdx.x / cluster_ctas();
  const int j = (int)(r % A.J), k = (int)(r / A.J % A.K);
  const long long b = r / A.J / A.K;
  float itf = sample_setting(A.inv_temp, b, k, j), p = sample_setting(A.top_p, b, k, j), mp = sample_setting(A.min_p, b, k, j);
  int kk = A.top_k.rows ? __ldg((const int*)A.top_k.rows + b * A.top_k.sb + k * A.top_k.sk + j * A.top_k.sj) : A.top_k.ivalue;
  const float u = __ldg(A.u + r);
  const bool greedy = itf == CUDART_INF_F;
  if (!((itf >= 1e-20f && itf <= 1e20f) || greedy) || !(p > 0.f) || !(mp >= 0.f && mp <= 1.f) || !(u >= 0.f && u <= 1.f)) {
    if (threadIdx.x == 0 && cluster_rank() == 0) {
      A.tokens[r] = -1;
      if (A.logprobs) A.logprobs[r] = 0.f;
      if (A.status) atomicOr(A.status, kSampleBadSetting);
    }
    return;
  }
  if (greedy) itf = 1.f, kk = 1;
  if (kk == 1) p = 1.f, mp = 0.f;
  const char* start = (const char*)A.data + (b * A.sb + k * A.sk + j * A.sj) * Row::ES;
  S.row.mis = (uint32_t)(((uintptr_t)start & 15) / Row::ES);
  S.row.base = start - S.row.mis * Row::ES;
  S.row.end = S.row.mis + (uint32_t)A.V;
  S.listed = -1;
  S.shift = A.shift;
  S.nch = (int)(((long long)S.row.end + (256LL << A.shift) - 1) >> (8 + A.shift));
  S.it = (double)itf;
  S.it2 = S.it * 1.4426950408889634;
  if (threadIdx.x < 16) sh.exp16[threadIdx.x] = exp2((double)threadIdx.x * 0.0625);
  const bool use_k = kk > 0 && kk < A.V, use_p = p < 1.f;
  const bool need_sum = !use_k && (use_p || mp == 0.f);
  const float c2 = (float)S.it2;
  if (cluster_ctas() > 1) {  // the first CTA's shared memory is written by the others
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  }
  if (need_sum) S.template sweep<true>(c2);
  else S.template sweep<false>(c2);
  if (cluster_ctas() > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (cluster_rank() != 0) return;
  }
  __syncthreads();
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
  S.set_top(m);
  typename Sampler<DT, THREADS>::Kept kept{-3.402823466e38f, m, S.row.end};
  // Relative error of the sweep's sums, were all roundings to go one way: exponentials 1.5e-7 (measured for every argument). Their
  // exponents t, 2^-24 |t| per rounding: two, the difference's and c2's own (the sets' references are set off against one another in
  // 64 bits), where |t|, weighted by the terms of 1024, is 6.4 at most on the mean (one term of 1, 1023 of 2^-7.85) and 0.5
  // more by the reference's rounding.  Ten additions, 2^-24 each.  Rows with many equal logits come near it: one token above
  // 152063 equal ones is off by 5e-7 by c2 alone where their sums are taken relative to the row's.  Odd sets and chunks beyond 256
  // tokens have three roundings per exponent, a mean that grows by one per doubling, and 64-bit additions.
  const double eps = 1.5e-7 + 5.97e-8 * (19.3 + 2.1 * A.shift);
  double total = 0.0;
  uint32_t pos = S.row.mis;
  bool done = false;
  if (need_sum) {
    for (int g = threadIdx.x; g < kSampleChunks; g += THREADS) {
      double y = 0.0;
      if (4 * g < S.nch) {
        const float mm = fmaxf(fmaxf(sh.cmax[4 * g], sh.cmax[4 * g + 1]), fmaxf(sh.cmax[4 * g + 2], sh.cmax[4 * g + 3]));
        if (mm > -CUDART_INF_F)
          y = (double)sh.csum[g] * exp2(((double)mm - (double)m) * S.it2 + (S.by_product(mm * c2) ? (double)(mm * c2) - (double)mm * (double)c2 : 0.0));
      }
      sh.psum[g] = y;
    }
    __syncthreads();
    // (the ends of the unit interval have tokens whose weights no sum may round away)
    if (!use_p && u > 0.f && u < 1.f) done = Calls::locate(S, kept, (double)u, 10 + A.shift, 1.01 * eps, &pos, &total);
  }
  if (!done) {
    // the least code that min-p keeps
    uint32_t floor_code = Row::kLowest;
    if (mp > 0.f) {
      const double ln = log((double)mp);
      float edge = (float)((double)m + ln / S.it);
      if (!(edge >= -3.402823466e38f)) edge = -3.402823466e38f;
      const uint32_t hi = Row::key(m);
      uint32_t e = min(Row::key(edge), hi);
      const auto keeps = [&](uint32_t c) { return ((double)Row::value(c) - (double)m) * S.it >= ln; };
      // The edge is off by its rounding, most often by no code or one.  Around zero codes lie far closer than the
      // 64-bit difference tells apart (a million of them for ordinary settings): there by halving.
      if (!keeps(e)) e = min(e + 1u, hi);
      if ((e < hi && !keeps(e)) || (e > Row::kLowest && keeps(e - 1u))) {
        uint32_t below = Row::kLowest;
        e = hi;  // always kept
        while (below < e) {
          const uint32_t c = below + (e - below) / 2u;
          if (keeps(c)) e = c;
          else below = c + 1u;
        }
      }
      floor_code = e;
    }
    uint32_t code = floor_code;         // the least kept one
    uint32_t take = 0u, equal = 0u;     // of the tokens that have it; equal == 0: all of them stay
    uint32_t pc, pt, pe;
    if (use_k) {
      // top-p needs the mass of all k
      const uint32_t lowest = use_p ? Row::kLowest : floor_code;
      // At least k tokens reach the k-th largest chunk maximum.  With more of them to keep than there are chunks, a
      // smaller one is taken that about 1.5 k tokens reach if they lie anywhere; where fewer than k do, one goes further down.
      const int nth = kk <= S.nch ? kk : max(1, min(S.nch, (int)((float)S.nch * (1.f - __expf(-1.5f * (float)kk / (float)S.nch)))));
      uint32_t cut = Calls::kth_chunk(S, (uint32_t)nth);
      bool limited = false;
      for (int tries = 0;; ++tries) {
        if (cut < lowest) cut = lowest;
        Calls::make_list(S, Row::value(cut));
        if (kk <= kSampleList / 3 * 2) S.listed = Calls::gather(S, Row::value(cut), m);  // +inf and NaN are masked
        if (S.listed >= 0 && S.listed <= THREADS && (S.listed >= kk || cut == lowest)) {
          Calls::pick(S, (uint32_t)kk, use_p, (double)p, floor_code, (double)u, &pos, &total);
          done = true;
          break;
        }
        limited = Calls::kth(S, cut, (uint32_t)kk, &code, &take, &equal);
        if (limited || cut == lowest) break;
        // Further down by half of the way so far, by a code at least (below 0 a bf16 code holds what lies less than a step below its
        // value); after eight times to the end, which rows with fewer than k tokens come to.
        const float v = Row::value(cut), further = v - (m - v) * 0.5f;
        cut = tries < 8 && further > -3.402823466e38f ? min(Row::key(further), cut - 1u) : lowest;
      }
      if (!limited) take = equal = 0u, code = cut;
      if (!done && use_p && Calls::nucleus(S, code, equal - take, true, false, (double)p, 0.0, 0.0, &pc, &pt, &pe) == 1) code = pc, take = pt, equal = pe;
    } else if (use_p) {
      double goal = S.total_mass(), slack = eps;
      uint32_t was = 0u;
      for (int pass = 0; pass < 2; ++pass) {
        // what lies below max - c has at most V e^(-c inv_temp) = (1 - p) total
        const double c = log((double)A.V / ((1.0 - (double)p) * goal * (1.0 - 2.0 * eps))) / S.it;
        float edge = (float)((double)m - (c > 0.0 ? c : 0.0) * (1.0 + 1e-6));
        if (!(edge >= -3.402823466e38f)) edge = -3.402823466e38f;
        uint32_t cut = Row::key(edge);
        if (cut > Row::kLowest) --cut;
        if (cut < floor_code) cut = floor_code;
        Calls::make_list(S, Row::value(cut));
        const int got = Calls::nucleus(S, cut, 0u, false, pass == 1 && cut == was && Row::key(m) - cut < (uint32_t)kSampleBins, 0.0, (double)p * goal * (1.0 - slack), (double)p * goal * (1.0 + slack), &pc, &pt, &pe);
        if (got == 1) code = pc, take = pt, equal = pe;
        else if (got == 0) code = cut;
        if (got >= 0) break;
        was = cut;
        // the border lies within the sweep's error: the total in 64 bits
        Calls::make_list(S, -3.402823466e38f);
        Calls::exact_sums(S, kept);
        goal = S.total_mass();
        slack = 0.0;
      }
    }
    if (code < floor_code) code = floor_code, take = equal = 0u;
    if (!done && S.listed < 0) {
      Calls::make_list(S, Row::value(code));
      if (use_k || use_p || mp > 0.f) S.listed = Calls::gather(S, Row::value(code), m);
    }
    if (!done && S.listed >= 0) {
      Calls::locate_listed(S, code, take < equal ? take : 0xffffffffu, (double)u, &pos, &total);
    } else if (!done) {
      kept.from = Row::value(code);
      if (take < equal) kept.end = Calls::equal_end(S, code, take);
      Calls::exact_sums(S, kept);
      Calls::locate(S, kept, (double)u, 8 + A.shift, 0.0, &pos, &total);
      if (!(u > 0.f && u < 1.f)) {  // the first or the last one that has a weight, by their number: weights of 1
        double number;
        S.it2 = 0.0;
        Calls::exact_sums(S, kept);
        Calls::locate(S, kept, (double)u, 8 + A.shift, 0.0, &pos, &number);
      }
    }
  }
  if (threadIdx.x == 0) {
    A.tokens[r] = (int32_t)(pos - S.row.mis);
    if (A.logprobs) {
      const float x = DT == kBF16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)S.row.base + pos) << 16)
                                  : __ldg((const float*)S.row.base + pos);
      // none is positive: a total of the sweep may be below 1 by its rounding
      A.logprobs[r] = fminf((float)(((double)x - (double)m) * S.it - log(total)), 0.f);
    }
  }
}

}  // namespace gls
