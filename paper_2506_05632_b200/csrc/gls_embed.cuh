// gls_embed.cuh -- rows of a table by token, scaled, and the gradient with respect to the table.
//
//   out[n] = scale * table[token[n]]                     (a token below 0 gives a row of zeros)
//   grad_table[v] = scale * sum over n with token[n] == v of grad_out[n]
//
// The gradient sorts the tokens (stable, so that equal tokens stay in the order of n), cuts the
// sorted positions into ranges of a fixed length and sums each range's rows in order; what a token
// has in more than one range is joined by a last kernel: in order for up to 32 ranges more, beyond that by
// eight warps, each every eighth range in order, whose sums are then added in turn.  The result does not
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
// What an earlier launch of the same call has written.  The launches overlap (see zero_share), so a grid may
// have started before these writes; the read-only path (__ldg) is for data that stays as it is while a grid
// lives and is not for them, a plain load behind griddepcontrol.wait sees them.
template <class T>
__device__ __forceinline__ T ld_made(const T* p) {
  static_assert(sizeof(T) == 4, "a word");
  uint32_t v;
  asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return (T)v;
}
template <int DT>
__device__ __forceinline__ uint32_t scale_word(uint32_t w, float s) {
  if (DT == kF32) return __float_as_uint(__uint_as_float(w) * s);
  return pack_bf16x2(bf16_lo(w) * s, bf16_hi(w) * s);
}

// ---- rows at any alignment -------------------------------------------------------------------
// Rows of an odd size start anywhere.  What is written is cut at 16-byte boundaries of the output; the 16
// bytes for one store are taken from the two aligned words of the source that hold them.  A word may reach
// into the row's neighbours, whose elements are not used, but not out of the tensor [lo, hi).
template <int ES>
__device__ __noinline__ uint4 span_edge(uintptr_t at, uintptr_t lo, uintptr_t hi) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uintptr_t p = at + 4 * i;
    if constexpr (ES == 4) {
      w[i] = p >= lo && p < hi ? __float_as_uint(__ldg((const float*)p)) : 0u;
    } else {
      const uint32_t a = p >= lo && p < hi ? (uint32_t)__ldg((const unsigned short*)p) : 0u;
      const uint32_t b = p + 2 >= lo && p + 2 < hi ? (uint32_t)__ldg((const unsigned short*)(p + 2)) : 0u;
      w[i] = a | (b << 16);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int ES>
__device__ __forceinline__ uint4 span_word(uintptr_t at, uintptr_t lo, uintptr_t hi) {
  if (at >= lo && at + 16 <= hi) return ld_global16((const void*)at);
  if (at + 16 <= lo || at >= hi) return make_uint4(0u, 0u, 0u, 0u);
  return span_edge<ES>(at, lo, hi);
}
// N 4-byte words that begin `by` bytes (0 .. 15, even) into N + 4 of them
template <int N>
__device__ __forceinline__ void shift_words(const uint32_t (&w)[N + 4], int by, uint32_t (&o)[N]) {
  uint32_t a[N + 2], b[N + 1];
#pragma unroll
  for (int i = 0; i < N + 2; ++i) a[i] = (by & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < N + 1; ++i) b[i] = (by & 4) ? a[i + 1] : a[i];
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = __funnelshift_r(b[i], b[i + 1], (by & 2) * 8);
}
// 16 bytes at offset `o` (which may stick out at either end) of a row of `len` bytes
template <int ES>
__device__ __forceinline__ void row_put16(char* row, long long o, long long len, uint4 v) {
  if (o >= 0 && o + 16 <= len) {
    *(uint4*)(row + o) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 16 / ES; ++e) {
    const long long at = o + e * ES;
    if (at < 0 || at >= len) continue;
    if constexpr (ES == 4) *(uint32_t*)(row + at) = w[e];
    else *(unsigned short*)(row + at) = (unsigned short)(w[e >> 1] >> (16 * (e & 1)));
  }
}
// 16-byte pieces that a row of `len` bytes can touch
__host__ __device__ __forceinline__ long long row_pieces(long long len, int es) { return (len + 16 - es + 15) / 16; }

constexpr int kEmbedThreads = 256;
constexpr int kEmbedUnits = 4;  // per thread, requested together
// Units of 16 bytes, `per_row` to a row; a CTA takes 1024 in a row.
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_vec_kernel(const __grid_constant__ EmbedArgs A, uint32_t per_row) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const long long n_units = A.N * per_row;
  for (long long u0 = (long long)blockIdx.x * (kEmbedThreads * kEmbedUnits) + threadIdx.x; u0 < n_units;
       u0 += (long long)gridDim.x * (kEmbedThreads * kEmbedUnits)) {
    uint4 v[kEmbedUnits];
    char* to[kEmbedUnits];
#pragma unroll
    for (int j = 0; j < kEmbedUnits; ++j) {
      const long long u = u0 + j * kEmbedThreads;
      v[j] = make_uint4(0u, 0u, 0u, 0u);
      to[j] = nullptr;
      if (u >= n_units) continue;
      const long long n = u < (1ll << 32) ? (long long)((uint32_t)u / per_row) : u / per_row;
      const long long c = (u - n * per_row) * 16;
      to[j] = A.out + n * A.out_stride * ES + c;
      const int t = __ldg(A.tokens + n);
      if (t >= 0 && t < A.V)
        v[j] = ld_global16(A.table + (long long)t * A.table_stride * ES + c);
      else if (t >= A.V && c == 0 && A.status != nullptr)
        atomicOr(A.status, kDevBadToken);
    }
#pragma unroll
    for (int j = 0; j < kEmbedUnits; ++j) {
      if (to[j] == nullptr) continue;
      if (A.scale != 1.0f) {
        v[j].x = scale_word<DT>(v[j].x, A.scale);
        v[j].y = scale_word<DT>(v[j].y, A.scale);
        v[j].z = scale_word<DT>(v[j].z, A.scale);
        v[j].w = scale_word<DT>(v[j].w, A.scale);
      }
      *(uint4*)to[j] = v[j];
    }
  }
}
// Rows of 64 units and more: a warp takes up to 128 units of one row, so that the division by the row
// length and the token are the warp's and not the unit's (65536 rows of 512 units: 138 -> 117 us).
constexpr uint32_t kEmbedLongRow = 64;
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_long_kernel(const __grid_constant__ EmbedArgs A, uint32_t per_row) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const int lane = threadIdx.x & 31;
  const uint32_t pieces = (per_row + 32 * kEmbedUnits - 1) / (32 * kEmbedUnits);
  const long long n_items = A.N * pieces;
  for (long long it = (long long)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5); it < n_items;
       it += (long long)gridDim.x * (kEmbedThreads / 32)) {
    const long long n = it < (1ll << 32) ? (long long)((uint32_t)it / pieces) : it / pieces;
    const uint32_t u0 = (uint32_t)(it - n * pieces) * (32 * kEmbedUnits) + lane;
    const int t = __ldg(A.tokens + n);
    const bool in = t >= 0 && t < A.V;
    if (t >= A.V && u0 == 0 && A.status != nullptr) atomicOr(A.status, kDevBadToken);
    const char* const from = A.table + (in ? (long long)t * A.table_stride * ES : 0ll);
    char* const to = A.out + n * A.out_stride * ES;
    uint4 v[kEmbedUnits];
#pragma unroll
    for (int j = 0; j < kEmbedUnits; ++j) {
      const uint32_t u = u0 + 32 * j;
      v[j] = make_uint4(0u, 0u, 0u, 0u);
      if (in && u < per_row) v[j] = ld_global16(from + (long long)u * 16);
    }
#pragma unroll
    for (int j = 0; j < kEmbedUnits; ++j) {
      const uint32_t u = u0 + 32 * j;
      if (u >= per_row) continue;
      if (in && A.scale != 1.0f) {
        v[j].x = scale_word<DT>(v[j].x, A.scale);
        v[j].y = scale_word<DT>(v[j].y, A.scale);
        v[j].z = scale_word<DT>(v[j].z, A.scale);
        v[j].w = scale_word<DT>(v[j].w, A.scale);
      }
      *(uint4*)(to + (long long)u * 16) = v[j];
    }
  }
}
// Any alignment, any D: a unit is one of the `per_row` 16-byte pieces that an output row can touch.  One
// element a thread instead took 535 us for 97450 rows of 1002 fp32.
template <int DT>
__device__ __forceinline__ uint4 embed_shifted(const uint32_t (&w)[8], int by, float scale, bool scaled) {
  uint32_t v[4];
  shift_words<4>(w, by, v);
  if (scaled) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = scale_word<DT>(v[i], scale);
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_shift_kernel(const __grid_constant__ EmbedArgs A, uint32_t per_row) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const long long len = A.D * ES;
  const uintptr_t lo = (uintptr_t)A.table, hi = lo + ((A.V - 1) * A.table_stride + A.D) * ES;
  const long long n_units = A.N * per_row;
  constexpr int kUnits = 2;  // in flight: 48 registers (300000 rows of 37 fp32 24 us; four of them, 76: 28)
  for (long long u0 = (long long)blockIdx.x * (kEmbedThreads * kEmbedUnits) + threadIdx.x; u0 < n_units;
       u0 += (long long)gridDim.x * (kEmbedThreads * kEmbedUnits)) {
#pragma unroll 1
    for (int half = 0; half < kEmbedUnits; half += kUnits) {
      uint32_t w[kUnits][8];
      long long o[kUnits];
      char* to[kUnits];
      int by[kUnits];
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        const long long it = u0 + (half + j) * kEmbedThreads;
        to[j] = nullptr;
        by[j] = -1;  // zeros
        o[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = 0u;
        if (it >= n_units) continue;
        const long long n = it < (1ll << 32) ? (long long)((uint32_t)it / per_row) : it / per_row;
        const uint32_t u = (uint32_t)(it - n * per_row);
        char* const row = A.out + n * A.out_stride * ES;
        o[j] = (long long)u * 16 - (long long)((uintptr_t)row & 15);
        if (o[j] >= len) continue;
        to[j] = row;
        const int t = __ldg(A.tokens + n);
        if (t >= 0 && t < A.V) {
          const uintptr_t q = lo + (uintptr_t)((long long)t * A.table_stride * ES + o[j]);
          by[j] = (int)(q & 15);
          const uint4 x = span_word<ES>(q - by[j], lo, hi);
          w[j][0] = x.x, w[j][1] = x.y, w[j][2] = x.z, w[j][3] = x.w;
          if (by[j] != 0) {
            const uint4 y = span_word<ES>(q - by[j] + 16, lo, hi);
            w[j][4] = y.x, w[j][5] = y.y, w[j][6] = y.z, w[j][7] = y.w;
          }
        } else if (t >= A.V && u == 0 && A.status != nullptr) {
          atomicOr(A.status, kDevBadToken);
        }
      }
#pragma unroll
      for (int j = 0; j < kUnits; ++j)
        if (to[j] != nullptr)
          row_put16<ES>(to[j], o[j], len, embed_shifted<DT>(w[j], max(by[j], 0), A.scale, by[j] >= 0 && A.scale != 1.0f));
    }
  }
}
// Long rows: a warp takes up to 128 units of one row, whose shift is the same for all of them (97450 rows of
// 1002 fp32 111 us; 65536 of 2283 bf16 148, and 192 with a row, an offset and a shift per unit).
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_shift_long_kernel(const __grid_constant__ EmbedArgs A, uint32_t per_row) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const int lane = threadIdx.x & 31;
  const long long len = A.D * ES;
  const uintptr_t lo = (uintptr_t)A.table, hi = lo + ((A.V - 1) * A.table_stride + A.D) * ES;
  const uint32_t pieces = (per_row + 32 * kEmbedUnits - 1) / (32 * kEmbedUnits);
  const long long n_items = A.N * pieces;
  for (long long it = (long long)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5); it < n_items;
       it += (long long)gridDim.x * (kEmbedThreads / 32)) {
    const long long n = it < (1ll << 32) ? (long long)((uint32_t)it / pieces) : it / pieces;
    const uint32_t u0 = (uint32_t)(it - n * pieces) * (32 * kEmbedUnits) + lane;
    char* const row = A.out + n * A.out_stride * ES;
    const long long o = (long long)u0 * 16 - (long long)((uintptr_t)row & 15);
    const int t = __ldg(A.tokens + n);
    const bool in = t >= 0 && t < A.V;
    if (t >= A.V && u0 == 0 && A.status != nullptr) atomicOr(A.status, kDevBadToken);
    const uintptr_t q = lo + (uintptr_t)((in ? (long long)t * A.table_stride * ES : 0ll) + o);
    const int by = (int)(q & 15);
    const bool scaled = in && A.scale != 1.0f;
    const uintptr_t from = q - by;
    constexpr long long kLast = 512 * (kEmbedUnits - 1);
    if (in && o >= 0 && o + kLast + 16 <= len && from >= lo && from + kLast + 32 <= hi) {
      uint32_t w[kEmbedUnits][8];
#pragma unroll
      for (int j = 0; j < kEmbedUnits; ++j) {
        const uint4 x = ld_global16((const void*)(from + 512 * j)), y = ld_global16((const void*)(from + 512 * j + 16));
        w[j][0] = x.x, w[j][1] = x.y, w[j][2] = x.z, w[j][3] = x.w;
        w[j][4] = y.x, w[j][5] = y.y, w[j][6] = y.z, w[j][7] = y.w;
      }
#pragma unroll
      for (int j = 0; j < kEmbedUnits; ++j) *(uint4*)(row + o + 512 * j) = embed_shifted<DT>(w[j], by, A.scale, scaled);
    } else {
#pragma unroll 1
      for (int j = 0; j < kEmbedUnits; ++j) {
        if (o + 512 * j >= len) break;
        uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
        if (in) {
          const uint4 x = span_word<ES>(from + 512 * j, lo, hi), y = span_word<ES>(from + 512 * j + 16, lo, hi);
          w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w, w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
        }
        row_put16<ES>(row, o + 512 * j, len, embed_shifted<DT>(w, by, A.scale, scaled));
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// gradient: rows of tokens that do not occur.  For a large table these zeros are most of what the call
// writes, and they depend on nothing but the tokens, so every launch below carries CTAs that write a
// share of them while its other CTAs, few and waiting on one another's results, leave the memory
// system idle.
// ------------------------------------------------------------------------------------------
enum : int { kZeroByBits, kZeroByTokens, kZeroByKeys };  // how a CTA learns which of its rows to leave
struct ZeroArgs {
  char* out;              // [V][D]
  long long out_stride;   // elements
  int V;
  long long D;
  int es;                 // bytes per element
  long long units;        // 16-byte pieces that a row can touch
  int how;
  const uint32_t* touched;  // by bits: one per token
  const int32_t* tokens;    // by tokens: the CTA looks through all of them
  const int32_t* keys;      // by keys: the sorted tokens; the CTA finds its own among them
  int N;
};
constexpr int kZeroRows = 16384;  // rows per CTA at most, except by bits

// `len` bytes from `p`, by the calling warp
__device__ __forceinline__ void zero_span(char* p, long long len, int es) {
  for (long long o = (long long)(threadIdx.x & 31) * 16 - (long long)((uintptr_t)p & 15); o < len; o += 512) {
    if (o >= 0 && o + 16 <= len) {
      *(uint4*)(p + o) = make_uint4(0u, 0u, 0u, 0u);
    } else {
      for (long long e = o < 0 ? 0 : o; e < len && e < o + 16; e += es) {
        if (es == 2) *(unsigned short*)(p + e) = 0;
        else *(float*)(p + e) = 0.f;
      }
    }
  }
}
// Rows [first, last) of tokens that do not occur, by the calling CTA.
__device__ __forceinline__ void zero_rows(const ZeroArgs& Z, long long first, long long last) {
  __shared__ uint32_t here[kZeroRows / 32];
  const bool look = Z.how != kZeroByBits;
  if (first >= last) return;
  if (look) {
    for (int w = threadIdx.x; w < (last - first + 31) / 32; w += blockDim.x) here[w] = 0u;
    __syncthreads();
    if (Z.how == kZeroByTokens) {
#pragma unroll 1
      for (int i0 = 0; i0 < Z.N; i0 += 8 * blockDim.x) {
        int t[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int i = i0 + q * blockDim.x + threadIdx.x;
          t[q] = i < Z.N ? __ldg(Z.tokens + i) : -1;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const long long r = (long long)t[q] - first;
          if (r >= 0 && r < last - first) atomicOr(&here[r >> 5], 1u << (r & 31));
        }
      }
    } else {
      // the first key that is not below `first`: the range is cut by as many threads at a time
      int lo = 0, n = Z.N;  // it is in [lo, lo + n]
      while (n > 0) {
        const int part = (n + (int)blockDim.x) / ((int)blockDim.x + 1);  // 1 .. n
        const int at = (int)(threadIdx.x + 1) * part - 1;                // the last of this thread's part
        const int below = __syncthreads_count(at < n && ld_made(Z.keys + lo + at) < first);
        lo += below * part;
        n = min(n - below * part, part - 1);
      }
      for (int i = lo + threadIdx.x; i < Z.N; i += blockDim.x) {
        const long long r = (long long)ld_made(Z.keys + i) - first;
        if (r >= last - first) break;
        atomicOr(&here[r >> 5], 1u << (r & 31));
      }
    }
    __syncthreads();
  }
  const int warps = (int)(blockDim.x >> 5);
  if (Z.out_stride == Z.D && last - first >= 4 * warps) {
    // Rows without gaps between them: each warp writes its rows' runs, whatever a row's size and alignment.
    const long long part = (last - first + warps - 1) / warps, base = look ? first : 0ll, row = Z.D * Z.es;
    const long long a = first + (threadIdx.x >> 5) * part, b = min(last, a + part);
    auto bits = [&](long long v) { return look ? here[(v - base) >> 5] : ld_made(Z.touched + (v >> 5)); };
    for (long long v = a; v < b;) {
      const int at = (int)((v - base) & 31);
      const uint32_t w = bits(v) >> at;
      if (w & 1u) {  // rows that occur
        v += min(~w != 0u ? __ffs(~w) - 1 : 32, 32 - at);
        continue;
      }
      long long e = v + (w != 0u ? __ffs(w) - 1 : 32 - at);
      while (w == 0u && e < b) {
        const uint32_t x = bits(e);
        e += x != 0u ? __ffs(x) - 1 : 32;
        if (x != 0u) break;
      }
      e = min(e, b);
      char* const from = Z.out + v * row;
      zero_span(from, (e - v) * row, Z.es);
      v = e;
    }
    return;
  }
  // rows side by side where one does not fill the CTA
  const long long units = Z.units, len = Z.D * Z.es;
  const int side = units < blockDim.x ? (int)(blockDim.x / (unsigned)units) : 1;
  const int mine = units < blockDim.x ? (int)(threadIdx.x / (unsigned)units) : 0;
  const long long c0 = units < blockDim.x ? (long long)(threadIdx.x % (unsigned)units) : (long long)threadIdx.x;
  if (mine >= side) return;
  for (long long v = first + mine; v < last; v += side) {
    const long long b = look ? v - first : v;
    if (((look ? here[b >> 5] : ld_made(Z.touched + (b >> 5))) >> (b & 31)) & 1u) continue;
    char* const row = Z.out + v * Z.out_stride * Z.es;
    const long long off = (long long)((uintptr_t)row & 15);
    for (long long o = c0 * 16 - off; o < len; o += 16ll * blockDim.x) {
      if (o >= 0 && o + 16 <= len) {
        *(uint4*)(row + o) = make_uint4(0u, 0u, 0u, 0u);
      } else {
        for (long long e = o < 0 ? 0 : o; e < len && e < o + 16; e += Z.es) {
          if (Z.es == 2) *(unsigned short*)(row + e) = 0;
          else *(float*)(row + e) = 0.f;
        }
      }
    }
  }
}
// A launch's share: rows [first, last) over CTAs `from` and up, `each` rows per CTA.
struct ZeroShare {
  long long first, last;
  int from, each;
};
// The launches of a call follow one another as programmatic dependents: every CTA lets the next launch
// start and then waits for the one before, except that CTAs which look through the tokens need nothing
// of it.  True for a CTA that has written its share.
__device__ __forceinline__ bool zero_share(const ZeroArgs& Z, const ZeroShare& h) {
  asm volatile("griddepcontrol.launch_dependents;");
  if ((int)blockIdx.x < h.from || Z.how != kZeroByTokens) asm volatile("griddepcontrol.wait;" ::: "memory");
  if ((int)blockIdx.x < h.from) return false;
  const long long a = h.first + (long long)(blockIdx.x - h.from) * h.each;
  zero_rows(Z, a, min(h.last, a + h.each));
  return true;
}

// ------------------------------------------------------------------------------------------
// gradient: the sort.  Least significant digit first; a tile of positions per CTA.
// cnt[pass][tile][digit] holds the tiles' digit counts of a pass; a pass places its keys from the
// counts and counts the next pass's digits at the places they went to.  Tokens outside [0, V) get
// the key V and end up behind the others.
// ------------------------------------------------------------------------------------------
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortMaxBits = 9;
constexpr int kSortBins = 1 << kSortMaxBits;
constexpr int kSortRounds = 4;                         // keys per thread
constexpr int kSortTile = kSortThreads * kSortRounds;  // 2048
// Tiles up to which every CTA of a pass adds up the others' counts itself; beyond, a launch per pass turns
// them into places first.
constexpr int kSortFewTiles = 64;

struct SortArgs {
  const int32_t* tokens;
  int N, V, bits, passes, tiles;
  uint32_t* cnt;                  // [passes][tiles][kSortBins]
  uint32_t* sum;                  // [passes][kSortBins]: where there are many tiles, the digits' totals
  uint32_t* touched;              // [(V + 31) / 32] bits, or NULL
  int32_t* key[2];                // ping, pong
  int32_t* pos[2];
  uint32_t* status;
  ZeroArgs zero;
};

__global__ void __launch_bounds__(kSortThreads) embed_sort_count_kernel(const __grid_constant__ SortArgs S) {
  __shared__ uint32_t h[kSortBins];
  asm volatile("griddepcontrol.launch_dependents;");
  for (int d = threadIdx.x; d < kSortBins; d += kSortThreads) h[d] = 0u;
  __syncthreads();
  const uint32_t mask = (1u << S.bits) - 1u;
  const int i0 = blockIdx.x * kSortTile;
  int t[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * kSortThreads + threadIdx.x;
    t[r] = i < S.N ? __ldg(S.tokens + i) : -1;
  }
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = i0 + r * kSortThreads + threadIdx.x;
    if (i >= S.N) continue;
    const int key = t[r] >= 0 && t[r] < S.V ? t[r] : S.V;
    atomicAdd(&h[key & mask], 1u);
    if (key < S.V) {
      if (S.touched != nullptr) atomicOr(S.touched + (key >> 5), 1u << (key & 31));
    } else if (t[r] >= S.V && S.status != nullptr) {
      atomicOr(S.status, kDevBadToken);
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kSortBins; d += kSortThreads) S.cnt[(long long)blockIdx.x * kSortBins + d] = h[d];
}

// Stable ranks of a tile's keys by digit: warp w owns 32 ROUNDS consecutive keys, 32 a round.  On
// return wc[w][d] is the number of keys with digit d before warp w in the tile, total[d] the tile's, and
// rank[r] the number before this one in its warp.
template <int ROUNDS, int WARPS, int BINS>
__device__ __forceinline__ void tile_ranks(const uint32_t (&digit)[ROUNDS], const bool (&valid)[ROUNDS],
                                           int (&rank)[ROUNDS], uint16_t (*wc)[BINS], uint32_t* total, int bins) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t lt = (1u << lane) - 1u;
  for (int d = lane; d < bins / 2; d += 32) ((uint32_t*)wc[warp])[d] = 0u;
  __syncwarp();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
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
  for (int d = threadIdx.x; d < bins; d += 32 * WARPS) {
    uint32_t c[WARPS], run = 0u;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) c[w] = wc[w][d];
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      wc[w][d] = (uint16_t)run;
      run += c[w];
    }
    total[d] = run;
  }
  __syncthreads();
}

// exclusive scan over the CTA's values (one per thread)
template <int WARPS>
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
    uint32_t s = lane < WARPS ? warp_sums[lane] : 0u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += o;
    }
    if (lane < WARPS) warp_sums[lane] = s;
  }
  __syncthreads();
  const uint32_t r = incl - x + (warp > 0 ? warp_sums[warp - 1] : 0u);
  __syncthreads();
  return r;
}

// Many tiles: the counts of a pass become, per digit, the sums over the tiles before each.  A CTA takes 32
// digits, its warps the tiles in contiguous parts.
constexpr int kScanWarps = 16;
__global__ void __launch_bounds__(32 * kScanWarps) embed_sort_scan_kernel(const __grid_constant__ SortArgs S, int pass) {
  __shared__ uint32_t part[kScanWarps][32];
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int d = (int)blockIdx.x * 32 + lane;
  uint32_t* const cnt = S.cnt + (long long)pass * S.tiles * kSortBins + d;
  const int each = (S.tiles + kScanWarps - 1) / kScanWarps;
  const int t0 = min(S.tiles, warp * each), t1 = min(S.tiles, t0 + each);
  uint32_t run = 0u;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) run += __ldcg(cnt + (long long)t * kSortBins);
  part[warp][lane] = run;
  __syncthreads();
  run = 0u;
  for (int w = 0; w < warp; ++w) run += part[w][lane];
  for (int t = t0; t < t1; ++t) {
    uint32_t* const p = cnt + (long long)t * kSortBins;
    const uint32_t c = __ldcg(p);
    __stcg(p, run);
    run += c;
  }
  if (warp == kScanWarps - 1) S.sum[pass * kSortBins + d] = run;
}

__global__ void __launch_bounds__(kSortThreads)
embed_sort_pass_kernel(const __grid_constant__ SortArgs S, int pass, const ZeroShare share) {
  __shared__ __align__(16) uint16_t wc[kSortWarps][kSortBins];
  __shared__ uint32_t base[kSortBins];
  __shared__ uint32_t warp_sums[kSortWarps], tile_total[kSortBins];
  static_assert(kSortBins == kSortThreads, "a thread per digit");
  if (zero_share(S.zero, share)) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t mask = (1u << S.bits) - 1u;
  const int shift = pass * S.bits;
  const uint32_t* cnt = S.cnt + (long long)pass * S.tiles * kSortBins;
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
      if (pass == 0) {
        const int t = __ldg(S.tokens + i);
        key[r] = t >= 0 && t < S.V ? t : S.V;
        pos[r] = i;
      } else {
        key[r] = __ldcg(kin + i);
        pos[r] = __ldcg(pin + i);
      }
    }
    digit[r] = ((uint32_t)key[r] >> shift) & mask;
  }
  // where this tile's keys of digit d = threadIdx.x start
  uint32_t total = 0u, before = 0u;
  if (S.tiles <= kSortFewTiles) {
#pragma unroll 8
    for (int t = 0; t < S.tiles; ++t) {
      const uint32_t c = __ldcg(cnt + (long long)t * kSortBins + threadIdx.x);
      if (t < (int)blockIdx.x) before += c;
      total += c;
    }
  } else {
    before = __ldcg(cnt + (long long)blockIdx.x * kSortBins + threadIdx.x);
    total = __ldcg(S.sum + pass * kSortBins + threadIdx.x);
  }
  base[threadIdx.x] = cta_scan<kSortWarps>(total, warp_sums) + before;
  tile_ranks<kSortRounds, kSortWarps, kSortBins>(digit, valid, rank, wc, tile_total, kSortBins);
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

// Fewer tokens: the whole sort in the first cluster of the launch, in its CTAs' shared memory; the other
// CTAs write zeros.  A CTA holds 2048 consecutive positions.  Per pass every CTA ranks its keys, the
// CTAs read one another's digit counts, and each key goes straight to its place in the shared memory of
// the CTA that holds it next.  (5000 tokens, 32000 x 64 bf16, the whole call: 18 us; with the kernels above
// 24.  Clusters of 16, which not every GPU can place, would take 20000 tokens in 26 us instead of 32; with
// 4096 positions per CTA 65536 tokens take 86 us where the kernels above take 71.)
constexpr int kClSortThreads = 1024;
constexpr int kClSortWarps = kClSortThreads / 32;
constexpr int kClSortCtas = 8;
constexpr int kClSortMaxBits = 10;
constexpr int kClSortBins = 1 << kClSortMaxBits;
constexpr int kClSortRounds = 2;     // keys per thread
constexpr int kClSortTile = kClSortThreads * kClSortRounds;
constexpr int kClSortMost = kClSortTile * kClSortCtas;  // 16384
struct ClSortShared {
  uint2 item[2][kClSortTile];  // (key, position)
  uint16_t wc[kClSortWarps][kClSortBins];
  uint32_t total[2][kClSortBins];
  uint32_t base[kClSortBins];
  uint32_t warp_sums[kClSortWarps];
};
static_assert(kClSortBins == kClSortThreads, "a thread per digit");

__global__ void __launch_bounds__(kClSortThreads)
embed_sort_cluster_kernel(const __grid_constant__ SortArgs S, int* counters, int ctas, const ZeroShare share) {
  if (zero_share(S.zero, share)) return;  // share.from == ctas: whole clusters
  extern __shared__ __align__(16) unsigned char score_smem[];
  ClSortShared& sh = *(ClSortShared*)score_smem;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = (int)blockIdx.x;
  const uint32_t mask = (1u << S.bits) - 1u;
  if (cta == 0 && tid < 2) counters[tid] = 0;
  uint32_t key[kClSortRounds], pos[kClSortRounds], digit[kClSortRounds];
  int rank[kClSortRounds];
  bool valid[kClSortRounds];
  const int i0 = warp * 32 * kClSortRounds + lane;  // within the tile
#pragma unroll
  for (int r = 0; r < kClSortRounds; ++r) {
    const int i = cta * kClSortTile + i0 + r * 32;
    valid[r] = i < S.N;
    key[r] = 0u;
    pos[r] = (uint32_t)i;
    if (valid[r]) {
      const int t = __ldg(S.tokens + i);
      key[r] = t >= 0 && t < S.V ? (uint32_t)t : (uint32_t)S.V;
      if (t >= S.V && S.status != nullptr) atomicOr(S.status, kDevBadToken);
    }
  }
  for (int pass = 0; pass < S.passes; ++pass) {
    const int shift = pass * S.bits, half = pass & 1;
#pragma unroll
    for (int r = 0; r < kClSortRounds; ++r) digit[r] = (key[r] >> shift) & mask;
    tile_ranks<kClSortRounds, kClSortWarps, kClSortBins>(digit, valid, rank, sh.wc, sh.total[half], (int)mask + 1);
    // all CTAs' counts are there, and all CTAs have read what the last pass left in `item`
    if (ctas > 1) {
      cluster_arrive();
      cluster_wait();
    }
    uint32_t before = 0u, all = 0u;
    if ((uint32_t)tid <= mask) {
      for (int c = 0; c < ctas; ++c) {
        const uint32_t n = cluster_ld32(cluster_map(&sh.total[half][tid], (uint32_t)c));
        if (c < cta) before += n;
        all += n;
      }
    }
    const uint32_t start = cta_scan<kClSortWarps>(all, sh.warp_sums) + before;
    sh.base[tid] = start;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kClSortRounds; ++r) {
      if (!valid[r]) continue;
      const uint32_t at = sh.base[digit[r]] + sh.wc[warp][digit[r]] + (uint32_t)rank[r];
      if (!GLS_IN_RANGE(at, 0, S.N, 71u)) continue;
      cluster_st64(cluster_map(&sh.item[half][at % kClSortTile], at / kClSortTile),
                   ((unsigned long long)pos[r] << 32) | key[r]);
    }
    if (ctas > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < kClSortRounds; ++r) {
      if (valid[r]) {
        const uint2 x = sh.item[half][i0 + r * 32];
        key[r] = x.x;
        pos[r] = x.y;
      }
    }
  }
  int32_t* const kout = S.key[(S.passes - 1) & 1];
  int32_t* const pout = S.pos[(S.passes - 1) & 1];
#pragma unroll
  for (int r = 0; r < kClSortRounds; ++r) {
    const int i = cta * kClSortTile + i0 + r * 32;
    if (valid[r]) {
      kout[i] = (int32_t)key[r];
      pout[i] = (int32_t)pos[r];
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
  float* partial;          // [2 * ranges][partial_stride]: columns as they lie in the token's row, see eg_first
  long long partial_stride;
  int* counters;           // [2]: heads that go on for a few ranges, for many
  int4* heads;             // [2][ranges]: range, token, ranges that go on with it (few)
  int N, V;
  long long D;
  int per_range, ranges, slabs, accumulate;
  float scale;
  ZeroArgs zero;
};

constexpr int kEgThreads = 256;
constexpr int kEgCols = 8;       // columns per thread
constexpr int kEgMaxRange = 64;  // sorted positions per range
constexpr int kEgBatch = 4;      // rows in flight
constexpr int kEgMany = 32;      // ranges from which a token's partials are shared out among warps

// A thread has eight neighbouring columns.  VEC: rows of a multiple of eight columns on 16-byte boundaries.
// Otherwise the columns are cut at the 16-byte boundaries of the token's row in the table, which begins
// eg_first columns behind one: what is written is aligned and what is read is shifted into place.
template <int DTO>
__device__ __forceinline__ int eg_first(const EmbedGradArgs& A, int token) {
  constexpr int ES = DTO == kBF16 ? 2 : 4;
  return (int)(((uintptr_t)A.out + (uintptr_t)((long long)token * A.out_stride * ES)) & 15) / ES;
}
__device__ __forceinline__ long long eg_place(int slab) { return ((long long)slab * blockDim.x + threadIdx.x) * kEgCols; }
template <int DT, bool VEC>
struct EgRow {
  static constexpr int kWords = DT == kBF16 ? 4 : 8;
  uint32_t w[kWords + (VEC ? 0 : 4)];
  int by;  // bytes that the columns begin behind w
};
// The words that hold the columns at `at[q]`; the tensor is [lo, hi).  All loads are on their way together.
template <int DT, bool VEC>
__device__ __forceinline__ void eg_load(EgRow<DT, VEC> (&r)[kEgBatch], const uintptr_t (&at)[kEgBatch], uintptr_t lo, uintptr_t hi) {
  constexpr int kLoads = (int)sizeof(r[0].w) / 16;
  bool inside = true;
#pragma unroll
  for (int q = 0; q < kEgBatch; ++q) {
    r[q].by = VEC ? 0 : (int)(at[q] & 15);
    inside = inside && at[q] - r[q].by >= lo && at[q] - r[q].by + 16 * kLoads <= hi;
  }
  auto put = [&](int q, int k, uint4 a) { r[q].w[4 * k] = a.x, r[q].w[4 * k + 1] = a.y, r[q].w[4 * k + 2] = a.z, r[q].w[4 * k + 3] = a.w; };
  if (VEC || inside) {
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q)
#pragma unroll
      for (int k = 0; k < kLoads; ++k) put(q, k, ld_global16((const void*)(at[q] - r[q].by + 16 * k)));
  } else {
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q)
#pragma unroll
      for (int k = 0; k < kLoads; ++k) put(q, k, span_word<DT == kBF16 ? 2 : 4>(at[q] - r[q].by + 16 * k, lo, hi));
  }
}
template <int DT, bool VEC>
__device__ __forceinline__ void eg_add(float (&acc)[kEgCols], const EgRow<DT, VEC>& r) {
  constexpr int kWords = EgRow<DT, VEC>::kWords;
  uint32_t v[kWords];
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) v[i] = r.w[i];
  } else {
    shift_words<kWords>(r.w, r.by, v);
  }
#pragma unroll
  for (int i = 0; i < kEgCols; ++i) {
    if constexpr (DT == kBF16) acc[i] += (i & 1) ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]);
    else acc[i] += __uint_as_float(v[i]);
  }
}
template <int DTO>
__device__ __forceinline__ void eg_write1(const EmbedGradArgs& A, int token, long long c, float sum) {
  char* const row = A.out + (long long)token * A.out_stride * (DTO == kBF16 ? 2 : 4);
  float v = sum * A.scale;
  if (A.accumulate) v += DTO == kF32 ? ((const float*)row)[c] : __uint_as_float((uint32_t)((const unsigned short*)row)[c] << 16);
  store_elem<DTO>(row, c, v);
}
template <int DTO, bool VEC>
__device__ __forceinline__ void eg_store(const EmbedGradArgs& A, int token, long long c, const float (&acc)[kEgCols]) {
  constexpr int ES = DTO == kBF16 ? 2 : 4;
  if (c >= A.D || c + kEgCols <= 0) return;
  if (!VEC && (c < 0 || c + kEgCols > A.D)) {
#pragma unroll
    for (int i = 0; i < kEgCols; ++i)
      if (c + i >= 0 && c + i < A.D) eg_write1<DTO>(A, token, c + i, acc[i]);
    return;
  }
  char* const row = A.out + (long long)token * A.out_stride * ES;
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
}

// CTAs [0, ranges * slabs): a range of sorted positions and a slab of columns each.  A token whose
// positions all lie in the range is written; what a range has of a token that began before it goes
// to the partial 2 r, of one that goes on behind it to 2 r + 1 (one that does both: 2 r), and a range
// in which a token begins that goes on is listed.
template <int DT, int DTO, bool VEC>
__global__ void __launch_bounds__(kEgThreads) embed_grad_kernel(const __grid_constant__ EmbedGradArgs A, const ZeroShare share) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  if (zero_share(A.zero, share)) return;
  __shared__ int sk[kEgMaxRange + 2], sp[kEgMaxRange];
  const int range = (int)(blockIdx.x / A.slabs), slab = (int)(blockIdx.x % A.slabs);
  const int i0 = range * A.per_range;
  const int n = min(A.per_range, A.N - i0);
  for (int i = threadIdx.x; i < n + 2; i += blockDim.x) {  // sk[0]: the key before the range, sk[n + 1]: behind it
    const int at = i0 + i - 1;
    sk[i] = at >= 0 && at < A.N ? ld_made(A.key + at) : -1;
    if (i >= 1 && i <= n) sp[i - 1] = ld_made(A.pos + at);
  }
  __syncthreads();
  if (slab == 0 && sk[n] < A.V && sk[n] == sk[n + 1] && sk[0] != sk[n]) {
    // how many ranges behind this one start with the token, up to kEgMany + 1
    int go = 0;
    for (int t0 = 0; t0 <= kEgMany; t0 += blockDim.x) {
      const int t = t0 + threadIdx.x;
      const long long at = (long long)i0 + (long long)(1 + t) * A.per_range;
      go += __syncthreads_count(t <= kEgMany && at < A.N && ld_made(A.key + at) == sk[n]);
    }
    if (threadIdx.x == 0) {
      const int many = go > kEgMany ? 1 : 0;
      // in any order: heads do not meet
      A.heads[(long long)many * A.ranges + atomicAdd(A.counters + many, 1)] = make_int4(range, sk[n], go, 0);
    }
  }
  const long long place = eg_place(slab);
  if (place >= A.partial_stride || sk[1] >= A.V) return;  // no column, only tokens outside the table
  const uintptr_t lo = (uintptr_t)A.g, hi = lo + ((A.N - 1ll) * A.g_stride + A.D) * ES;
  float acc[kEgCols];
#pragma unroll
  for (int i = 0; i < kEgCols; ++i) acc[i] = 0.f;
  bool from_before = sk[1] == sk[0];
  for (int i = 0; i < n; i += kEgBatch) {
    EgRow<DT, VEC> rows[kEgBatch];
    uintptr_t at[kEgBatch];
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q) {
      const int p = min(i + q, n - 1);  // behind the range and outside the table: any row, not used
      long long c = place - (VEC ? 0 : eg_first<DTO>(A, sk[p + 1]));
      if (!VEC && (c >= A.D || c + kEgCols <= 0)) c = 0;  // no column of this token: not used
      at[q] = lo + (uintptr_t)(((long long)sp[p] * A.g_stride + c) * ES);
    }
    eg_load<DT, VEC>(rows, at, lo, hi);
#pragma unroll
    for (int q = 0; q < kEgBatch; ++q) {
      if (i + q >= n) break;
      const int key = sk[i + q + 1];
      if (key >= A.V) return;  // only tokens outside the table from here on
      eg_add<DT, VEC>(acc, rows[q]);
      if (sk[i + q + 2] != key || i + q + 1 == n) {  // the token's last position here
        const bool goes_on = sk[i + q + 2] == key;
        if (!from_before && !goes_on) {
          eg_store<DTO, VEC>(A, key, place - (VEC ? 0 : eg_first<DTO>(A, key)), acc);
        } else if (place < A.partial_stride) {
          float* const p = A.partial + (2ll * range + (from_before ? 0 : 1)) * A.partial_stride + place;
          *(float4*)p = make_float4(acc[0], acc[1], acc[2], acc[3]);
          *(float4*)(p + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        }
        from_before = false;
#pragma unroll
        for (int c = 0; c < kEgCols; ++c) acc[c] = 0.f;
      }
    }
  }
}

// Joins the partials of the tokens that begin in a listed range and go on behind it: partial 2 r + 1
// of that range, then 2 r of each range after it that starts with the token.  Work items: for heads of
// a few ranges (head, four columns per thread); for heads of many (head, four columns per lane), whose
// ranges the CTA's eight warps share out, each adding its own in order.
struct EgVec {
  float v[4];
};
__device__ __forceinline__ EgVec eg_partial(const float* p) {
  EgVec x;
  asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x.v[0]), "=f"(x.v[1]), "=f"(x.v[2]), "=f"(x.v[3]) : "l"(p));
  return x;
}
// Four CTAs an SM leave a thread the registers for its eight loads; with the compiler's own choice of 40
// the join of 5536 tokens' rows of 480 fp32 takes 11 us instead of 9.
template <int DTO>
__global__ void __launch_bounds__(kEgThreads, 4) embed_join_kernel(const __grid_constant__ EmbedGradArgs A, const ZeroShare share) {
  if (zero_share(A.zero, share)) return;
  constexpr int W = 4;
  __shared__ float sums[kEgThreads][W];
  constexpr int kWarps = kEgThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long places = A.partial_stride;
  const uint32_t wide = (uint32_t)((places + W * kEgThreads - 1) / (W * kEgThreads)), narrow = (uint32_t)((places + W * 32 - 1) / (W * 32));
  const long long n_few = (long long)A.counters[0] * wide, n_items = n_few + (long long)A.counters[1] * narrow;
  for (long long it = blockIdx.x; it < n_items; it += share.from) {
    const bool many = it >= n_few;
    const long long i = many ? it - n_few : it;
    const uint32_t tiles = many ? narrow : wide;
    const int head = (int)(i / tiles);
    const long long c = ((i - (long long)head * tiles) * (many ? 32 : kEgThreads) + (many ? lane : (int)threadIdx.x)) * W;
    const int4 h = A.heads[(many ? A.ranges : 0) + head];
    int go = h.z;
    if (many) {
      for (;;) {
        const long long at = ((long long)h.x + 1 + go + threadIdx.x) * A.per_range;
        const int more = __syncthreads_count(at < A.N && ld_made(A.key + at) == h.y);
        go += more;
        if (more < kEgThreads) break;
      }
    }
    const int skip = eg_first<DTO>(A, h.y);  // place c is column c - skip
    const bool on = c < places;
    const int from = many ? warp : 0, step = many ? kWarps : 1;
    const long long cc = on ? c : 0;
    EgVec acc = eg_partial(A.partial + (2ll * h.x + 1) * places + cc);
    if (from != 0) acc = {{0.f, 0.f, 0.f, 0.f}};
    const float* const p = A.partial + 2ll * (h.x + 1) * places + cc;
    for (int r = from; r < go; r += 8 * step) {
      EgVec x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = eg_partial(p + 2ll * min(r + q * step, go - 1) * places);
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int e = 0; e < W; ++e) acc.v[e] += r + q * step < go ? x[q].v[e] : 0.f;
    }
    if (many) {
#pragma unroll
      for (int e = 0; e < W; ++e) sums[threadIdx.x][e] = acc.v[e];
      __syncthreads();
      if (warp == 0)
        for (int w = 1; w < kWarps; ++w)
#pragma unroll
          for (int e = 0; e < W; ++e) acc.v[e] += sums[w * 32 + lane][e];
      __syncthreads();
    }
    if (on && (!many || warp == 0)) {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (c + e >= skip && c + e - skip < A.D) eg_write1<DTO>(A, h.y, c + e - skip, acc.v[e]);
    }
  }
}

}  // namespace gls
