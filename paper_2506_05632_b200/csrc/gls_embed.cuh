// gls_embed.cuh -- rows of a table by token, scaled, and the gradient with respect to the table.
//
//   out[n] = scale * table[token[n]]                     (a token below 0 gives a row of zeros)
//   grad_table[v] = scale * sum over n with token[n] == v of grad_out[n]
//
// The gradient sorts the tokens (stable, so that equal tokens stay in the order of n), cuts the
// sorted positions into ranges of a fixed length and sums each range's rows in order; what a token
// has in more than one range is joined by a last kernel, again in order.  The result does not
// depend on how the blocks are scheduled, and a token that fills half the batch costs no more than
// many different ones.
#pragma once
#include "gls_logprob.cuh"

namespace gls {

// ------------------------------------------------------------------------------------------
// lookup
// ------------------------------------------------------------------------------------------
struct EmbedArgs {
  const char* table;
  long long table_stride;  // elements
  char* out;
  long long out_stride;
  const int32_t* tokens;
  long long N, V, D;
  float scale;
  uint32_t* status;
};

__device__ __forceinline__ uint4 ld_global16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
template <int DT>
__device__ __forceinline__ uint32_t scale_word(uint32_t w, float s) {
  if (DT == kF32) return __float_as_uint(__uint_as_float(w) * s);
  return pack_bf16x2(bf16_lo(w) * s, bf16_hi(w) * s);
}

constexpr int kEmbedThreads = 256;
// 16 bytes per unit; rows of `per_row` units
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_vec_kernel(const __grid_constant__ EmbedArgs A, int per_row) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const long long n_units = A.N * per_row;
  for (long long u = (long long)blockIdx.x * kEmbedThreads + threadIdx.x; u < n_units;
       u += (long long)gridDim.x * kEmbedThreads) {
    const long long n = u / per_row;
    const long long c = (u - n * per_row) * 16;
    const int t = __ldg(A.tokens + n);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (t >= 0 && t < A.V) {
      v = ld_global16(A.table + (long long)t * A.table_stride * ES + c);
      if (A.scale != 1.0f) {
        v.x = scale_word<DT>(v.x, A.scale);
        v.y = scale_word<DT>(v.y, A.scale);
        v.z = scale_word<DT>(v.z, A.scale);
        v.w = scale_word<DT>(v.w, A.scale);
      }
    } else if (t >= A.V && c == 0 && A.status != nullptr) {
      atomicOr(A.status, kDevBadToken);
    }
    *(uint4*)(A.out + n * A.out_stride * ES + c) = v;
  }
}
// any alignment, any D
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_any_kernel(const __grid_constant__ EmbedArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const long long n_units = A.N * A.D;
  for (long long u = (long long)blockIdx.x * kEmbedThreads + threadIdx.x; u < n_units;
       u += (long long)gridDim.x * kEmbedThreads) {
    const long long n = u / A.D;
    const long long c = u - n * A.D;
    const int t = __ldg(A.tokens + n);
    float x = 0.f;
    if (t >= 0 && t < A.V)
      x = load_logit<DT>(A.table + (long long)t * A.table_stride * ES, c) * A.scale;
    else if (t >= A.V && c == 0 && A.status != nullptr)
      atomicOr(A.status, kDevBadToken);
    store_elem<DT>(A.out + n * A.out_stride * ES, c, x);
  }
}

// ------------------------------------------------------------------------------------------
// gradient: the sort.  Least significant digit first; a tile of kSortTile positions per CTA.
// cnt[pass][tile][digit] holds the tiles' digit counts of a pass; a pass places its keys from the
// counts and counts the next pass's digits at the places they went to.  Tokens outside [0, V) get
// the key V and end up behind the others.
// ------------------------------------------------------------------------------------------
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortRounds = 8;                            // keys per lane
constexpr int kSortTile = kSortThreads * kSortRounds;     // 4096
constexpr int kSortMaxBits = 9;
constexpr int kSortBins = 1 << kSortMaxBits;

struct SortArgs {
  const int32_t* tokens;
  int N, V, bits, passes, tiles;
  uint32_t* cnt;                  // [passes][tiles][kSortBins]
  uint32_t* touched;              // [(V + 31) / 32] bits
  int32_t* key[2];                // ping, pong
  int32_t* pos[2];
  uint32_t* status;
};

__device__ __forceinline__ int sort_key(const SortArgs& S, int i) {
  const int t = __ldg(S.tokens + i);
  return t >= 0 && t < S.V ? t : S.V;
}

__global__ void __launch_bounds__(kSortThreads) embed_sort_count_kernel(const __grid_constant__ SortArgs S) {
  __shared__ uint32_t h[kSortBins];
  for (int d = threadIdx.x; d < kSortBins; d += kSortThreads) h[d] = 0u;
  __syncthreads();
  const uint32_t mask = (1u << S.bits) - 1u;
  const int i0 = blockIdx.x * kSortTile;
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * kSortThreads + threadIdx.x;
    if (i < S.N) {
      const int t = __ldg(S.tokens + i);
      const int key = t >= 0 && t < S.V ? t : S.V;
      atomicAdd(&h[key & mask], 1u);
      if (key < S.V) {
        const uint32_t bit = 1u << (key & 31);
        if (!(*(volatile uint32_t*)(S.touched + (key >> 5)) & bit)) atomicOr(S.touched + (key >> 5), bit);
      } else if (t >= S.V && S.status != nullptr) {
        atomicOr(S.status, kDevBadToken);
      }
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kSortBins; d += kSortThreads) S.cnt[(long long)blockIdx.x * kSortBins + d] = h[d];
}

// Stable ranks of a tile's keys by digit: warp w owns 256 consecutive keys, in rounds of 32.
// On return wc[w][d] is the number of keys with digit d before warp w in the tile and rank[r] the
// number before this one in its warp.
__device__ __forceinline__ void tile_ranks(const uint32_t (&digit)[kSortRounds], const bool (&valid)[kSortRounds],
                                           int (&rank)[kSortRounds], uint16_t (*wc)[kSortBins]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t lt = (1u << lane) - 1u;
  for (int d = lane; d < kSortBins; d += 32) wc[warp][d] = 0;
  __syncwarp();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const uint32_t d = valid[r] ? digit[r] : 0xffffffffu;
    const unsigned peers = __match_any_sync(0xffffffffu, d);
    int before = 0;
    if (valid[r]) before = wc[warp][d];
    __syncwarp();
    rank[r] = before + __popc(peers & lt);
    if (valid[r] && (peers & lt) == 0u) wc[warp][d] = (uint16_t)(before + __popc(peers));
    __syncwarp();
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kSortBins; d += kSortThreads) {
    uint32_t run = 0u;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = wc[w][d];
      wc[w][d] = (uint16_t)run;
      run += c;
    }
  }
  __syncthreads();
}

// exclusive scan over the CTA's kSortThreads values (one per thread)
__device__ __forceinline__ uint32_t cta_scan(uint32_t x, uint32_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    uint32_t s = lane < kSortWarps ? warp_sums[lane] : 0u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += o;
    }
    if (lane < kSortWarps) warp_sums[lane] = s;
  }
  __syncthreads();
  const uint32_t r = incl - x + (warp > 0 ? warp_sums[warp - 1] : 0u);
  __syncthreads();
  return r;
}

__global__ void __launch_bounds__(kSortThreads) embed_sort_pass_kernel(const __grid_constant__ SortArgs S, int pass) {
  __shared__ uint16_t wc[kSortWarps][kSortBins];
  __shared__ uint32_t base[kSortBins];
  __shared__ uint32_t warp_sums[kSortWarps];
  static_assert(kSortBins == kSortThreads, "a thread per digit");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t mask = (1u << S.bits) - 1u;
  const int shift = pass * S.bits;
  const uint32_t* cnt = S.cnt + (long long)pass * S.tiles * kSortBins;
  // where this tile's keys of digit d = threadIdx.x start
  uint32_t total = 0u, before = 0u;
  for (int t = 0; t < S.tiles; ++t) {
    const uint32_t c = __ldcg(cnt + (long long)t * kSortBins + threadIdx.x);
    if (t < (int)blockIdx.x) before += c;
    total += c;
  }
  base[threadIdx.x] = cta_scan(total, warp_sums) + before;

  const int32_t* kin = S.key[(pass + 1) & 1];
  const int32_t* pin = S.pos[(pass + 1) & 1];
  int32_t* kout = S.key[pass & 1];
  int32_t* pout = S.pos[pass & 1];
  int key[kSortRounds], pos[kSortRounds], rank[kSortRounds];
  uint32_t digit[kSortRounds];
  bool valid[kSortRounds];
  const int i0 = blockIdx.x * kSortTile + warp * 32 * kSortRounds;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * 32 + lane;
    valid[r] = i < S.N;
    key[r] = pos[r] = 0;
    if (valid[r]) {
      key[r] = pass == 0 ? sort_key(S, i) : __ldcg(kin + i);
      pos[r] = pass == 0 ? i : __ldcg(pin + i);
    }
    digit[r] = ((uint32_t)key[r] >> shift) & mask;
  }
  tile_ranks(digit, valid, rank, wc);
  uint32_t* next = pass + 1 < S.passes ? S.cnt + (long long)(pass + 1) * S.tiles * kSortBins : nullptr;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (!valid[r]) continue;
    const uint32_t at = base[digit[r]] + wc[warp][digit[r]] + (uint32_t)rank[r];
    if (!GLS_IN_RANGE(at, 0, S.N, 70u)) continue;
    kout[at] = key[r];
    pout[at] = pos[r];
    if (next != nullptr)
      atomicAdd(next + (long long)(at / kSortTile) * kSortBins + (((uint32_t)key[r] >> (shift + S.bits)) & mask), 1u);
  }
}

// At most kSortTile tokens: the whole sort in one CTA, through shared memory.
__global__ void __launch_bounds__(kSortThreads) embed_sort_small_kernel(const __grid_constant__ SortArgs S) {
  extern __shared__ __align__(16) unsigned char score_smem[];
  uint16_t(*wc)[kSortBins] = (uint16_t(*)[kSortBins])score_smem;
  int32_t* skey = (int32_t*)(score_smem + sizeof(uint16_t) * kSortWarps * kSortBins);
  uint16_t* spos = (uint16_t*)(skey + kSortTile);  // positions are below kSortTile
  __shared__ uint32_t base[kSortBins];
  __shared__ uint32_t warp_sums[kSortWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t mask = (1u << S.bits) - 1u;
  for (int w = threadIdx.x; w < (S.V + 31) / 32; w += kSortThreads) S.touched[w] = 0u;
  __syncthreads();
  int key[kSortRounds], pos[kSortRounds], rank[kSortRounds];
  uint32_t digit[kSortRounds];
  bool valid[kSortRounds];
  const int i0 = warp * 32 * kSortRounds;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * 32 + lane;
    valid[r] = i < S.N;
    key[r] = 0;
    pos[r] = i;
    if (valid[r]) {
      const int t = __ldg(S.tokens + i);
      key[r] = t >= 0 && t < S.V ? t : S.V;
      if (key[r] < S.V)
        atomicOr(S.touched + (key[r] >> 5), 1u << (key[r] & 31));
      else if (t >= S.V && S.status != nullptr)
        atomicOr(S.status, kDevBadToken);
    }
  }
  for (int pass = 0; pass < S.passes; ++pass) {
    const int shift = pass * S.bits;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) digit[r] = ((uint32_t)key[r] >> shift) & mask;
    tile_ranks(digit, valid, rank, wc);
    // keys of each digit in the whole tile: those before the last warp plus the last warp's own
    uint32_t* const hist = base;
    hist[threadIdx.x] = 0u;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (valid[r]) atomicAdd(&hist[digit[r]], 1u);
    __syncthreads();
    const uint32_t total = hist[threadIdx.x];
    const uint32_t start = cta_scan(total, warp_sums);
    base[threadIdx.x] = start;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      if (!valid[r]) continue;
      const uint32_t at = base[digit[r]] + wc[warp][digit[r]] + (uint32_t)rank[r];
      if (!GLS_IN_RANGE(at, 0, kSortTile, 71u)) continue;
      skey[at] = key[r];
      spos[at] = (uint16_t)pos[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      const int i = i0 + r * 32 + lane;
      if (valid[r]) {
        key[r] = skey[i];
        pos[r] = spos[i];
      }
    }
    __syncthreads();
  }
  int32_t* kout = S.key[(S.passes - 1) & 1];
  int32_t* pout = S.pos[(S.passes - 1) & 1];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * 32 + lane;
    if (valid[r]) {
      kout[i] = key[r];
      pout[i] = pos[r];
    }
  }
}

// ------------------------------------------------------------------------------------------
// gradient: the sums
// ------------------------------------------------------------------------------------------
struct EmbedGradArgs {
  const char* g;           // [N][D]
  long long g_stride;
  char* out;               // [V][D]
  long long out_stride;
  const int32_t* key;      // sorted tokens
  const int32_t* pos;      // their positions
  const uint32_t* touched;
  float* partial;          // [2 * ranges][D]
  int N, V;
  long long D;
  int per_range, ranges, slabs, accumulate;
  int zero_ctas;           // CTAs that write the rows of tokens that do not occur
  float scale;
};

constexpr int kEgCols = 8;       // columns per thread
constexpr int kEgMaxRange = 64;  // sorted positions per range
constexpr int kEgBatch = 4;      // rows in flight

// Columns of thread t in slab s: VEC: 8 neighbouring ones; otherwise every blockDim-th.
template <bool VEC>
__device__ __forceinline__ long long eg_col(int slab, int i) {
  const long long c0 = (long long)slab * blockDim.x * kEgCols;
  return VEC ? c0 + (long long)threadIdx.x * kEgCols + i : c0 + (long long)i * blockDim.x + threadIdx.x;
}
template <int DT, bool VEC>
struct EgRow {
  uint32_t w[VEC && DT == kBF16 ? 4 : 8];
};
template <int DT, bool VEC>
__device__ __forceinline__ void eg_load(EgRow<DT, VEC>& r, const char* row, int slab, long long D) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  if constexpr (VEC) {
    const long long c = eg_col<true>(slab, 0);
    if (c < D) {
      const uint4 a = ld_global16(row + c * ES);
      r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
      if constexpr (DT == kF32) {
        const uint4 b = ld_global16(row + c * ES + 16);
        r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEgCols; ++i) {
      const long long c = eg_col<false>(slab, i);
      r.w[i] = c < D ? __float_as_uint(load_logit<DT>(row, c)) : 0u;
    }
  }
}
template <int DT, bool VEC>
__device__ __forceinline__ float eg_get(const EgRow<DT, VEC>& r, int i) {
  if constexpr (VEC && DT == kBF16)
    return (i & 1) ? bf16_hi(r.w[i >> 1]) : bf16_lo(r.w[i >> 1]);
  else
    return __uint_as_float(r.w[i]);
}
template <int DTO, bool VEC>
__device__ __forceinline__ void eg_store(const EmbedGradArgs& A, int token, int slab, const float (&acc)[kEgCols]) {
  constexpr int ES = DTO == kBF16 ? 2 : 4;
  char* const row = A.out + (long long)token * A.out_stride * ES;
  if constexpr (VEC) {
    const long long c = eg_col<true>(slab, 0);
    if (c >= A.D) return;
    float v[kEgCols];
#pragma unroll
    for (int i = 0; i < kEgCols; ++i) v[i] = acc[i] * A.scale;
    uint4* const o = (uint4*)(row + c * ES);
    if constexpr (DTO == kBF16) {
      if (A.accumulate) {
        const uint4 x = *o;
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[2 * i] += bf16_lo(xw[i]);
          v[2 * i + 1] += bf16_hi(xw[i]);
        }
      }
      *o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4* const of = (float4*)o + h;
        float4 x = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
        if (A.accumulate) {
          const float4 y = *of;
          x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
        }
        *of = x;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEgCols; ++i) {
      const long long c = eg_col<false>(slab, i);
      if (c >= A.D) continue;
      float v = acc[i] * A.scale;
      if (A.accumulate) v += DTO == kF32 ? ((const float*)row)[c] : __uint_as_float((uint32_t)((const unsigned short*)row)[c] << 16);
      store_elem<DTO>(row, c, v);
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void eg_put(float* p, int slab, long long D, const float (&acc)[kEgCols]) {
#pragma unroll
  for (int i = 0; i < kEgCols; ++i) {
    const long long c = eg_col<VEC>(slab, i);
    if (c < D) p[c] = acc[i];
  }
}

// CTAs [0, ranges * slabs): a range of sorted positions and a slab of columns each.  A token whose
// positions all lie in the range is written; what a range has of a token that began before it goes
// to the partial 2 r, of one that goes on behind it to 2 r + 1 (one that does both: 2 r).
// The other CTAs write zeros to the rows of tokens that do not occur.
template <int DT, int DTO, bool VEC>
__global__ void __launch_bounds__(256) embed_grad_kernel(const __grid_constant__ EmbedGradArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  constexpr int ESO = DTO == kBF16 ? 2 : 4;
  const long long n_sum = (long long)A.ranges * A.slabs;
  if (blockIdx.x >= n_sum) {
    const long long rows_each = ((long long)A.V + A.zero_ctas - 1) / A.zero_ctas;
    const long long first = ((long long)blockIdx.x - n_sum) * rows_each;
    const long long last = min((long long)A.V, first + rows_each);
    for (long long v = first; v < last; ++v) {
      if ((__ldg(A.touched + (v >> 5)) >> (v & 31)) & 1u) continue;
      char* const row = A.out + v * A.out_stride * ESO;
      if constexpr (VEC) {
        for (long long c = (long long)threadIdx.x * 16; c < A.D * ESO; c += (long long)blockDim.x * 16)
          *(uint4*)(row + c) = make_uint4(0u, 0u, 0u, 0u);
      } else {
        for (long long c = threadIdx.x; c < A.D; c += blockDim.x) store_elem<DTO>(row, c, 0.f);
      }
    }
    return;
  }
  __shared__ int sk[kEgMaxRange + 2], sp[kEgMaxRange];
  const int range = (int)(blockIdx.x / A.slabs), slab = (int)(blockIdx.x % A.slabs);
  const int i0 = range * A.per_range;
  const int n = min(A.per_range, A.N - i0);
  for (int i = threadIdx.x; i < n + 2; i += blockDim.x) {  // sk[0]: the key before the range, sk[n + 1]: behind it
    const int at = i0 + i - 1;
    sk[i] = at >= 0 && at < A.N ? __ldg(A.key + at) : -1;
    if (i >= 1 && i <= n) sp[i - 1] = __ldg(A.pos + at);
  }
  __syncthreads();
  float acc[kEgCols];
#pragma unroll
  for (int i = 0; i < kEgCols; ++i) acc[i] = 0.f;
  bool from_before = sk[1] == sk[0];
  for (int i = 0; i < n; i += kEgBatch) {
    EgRow<DT, VEC> rows[kEgBatch];
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q)
      if (i + q < n && sk[i + q + 1] < A.V) eg_load<DT, VEC>(rows[q], A.g + (long long)sp[i + q] * A.g_stride * ES, slab, A.D);
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q) {
      if (i + q >= n) break;
      const int key = sk[i + q + 1];
      if (key >= A.V) return;  // only tokens outside the table from here on
#pragma unroll
      for (int c = 0; c < kEgCols; ++c) acc[c] += eg_get<DT, VEC>(rows[q], c);
      if (sk[i + q + 2] != key || i + q + 1 == n) {  // the token's last position here
        const bool goes_on = sk[i + q + 2] == key;
        if (from_before || goes_on)
          eg_put<VEC>(A.partial + (2ll * range + (from_before ? 0 : 1)) * A.D, slab, A.D, acc);
        else
          eg_store<DTO, VEC>(A, key, slab, acc);
        from_before = false;
#pragma unroll
        for (int c = 0; c < kEgCols; ++c) acc[c] = 0.f;
      }
    }
  }
}

// Joins the partials of the token that begins in a range and goes on behind it.
template <int DTO, bool VEC>
__global__ void __launch_bounds__(256) embed_join_kernel(const __grid_constant__ EmbedGradArgs A) {
  const int range = (int)(blockIdx.x / A.slabs), slab = (int)(blockIdx.x % A.slabs);
  const int i1 = (range + 1) * A.per_range;  // first position behind the range
  if (i1 >= A.N) return;
  const int key = __ldg(A.key + i1 - 1);
  if (key >= A.V || __ldg(A.key + i1) != key) return;
  const int i0 = range * A.per_range;
  if (i0 > 0 && __ldg(A.key + i0 - 1) == key) return;  // it began before: an earlier range joins it
  float acc[kEgCols];
#pragma unroll
  for (int i = 0; i < kEgCols; ++i) {
    const long long c = eg_col<VEC>(slab, i);
    acc[i] = c < A.D ? A.partial[(2ll * range + 1) * A.D + c] : 0.f;
  }
  for (int r = range + 1; r < A.ranges; ++r) {
#pragma unroll
    for (int i = 0; i < kEgCols; ++i) {
      const long long c = eg_col<VEC>(slab, i);
      if (c < A.D) acc[i] += A.partial[2ll * r * A.D + c];
    }
    const int next = (r + 1) * A.per_range;
    if (next >= A.N || __ldg(A.key + next) != key) break;
  }
  eg_store<DTO, VEC>(A, key, slab, acc);
}

}  // namespace gls
