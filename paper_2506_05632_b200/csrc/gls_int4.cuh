// gls_int4.cuh -- a table of V rows of D columns at 4 bits with a step (and a zero) per group of columns:
//     element (v, d) = scale[v, d / group] * (code[v, d] - zero[v, d / group])      zero 8 where none are given
// made from weights, read back by token, and multiplied with hidden states (the logits of a 4-bit head).
// Two codes a byte, the even column in the low half; a row's codes start on a 16-byte boundary.
#pragma once
#include <cuda.h>

#include "gls_async.cuh"
#include "gls_kernels.cuh"

namespace gls {

struct Int4Table {
  uint8_t* codes;          // [V] rows of code_stride bytes
  long long code_stride;
  void* scales;            // [V][G] fp32 or bf16
  long long scale_stride;  // elements
  uint8_t* zeros;          // NULL or [V][G]
  long long zero_stride;
  long long V, D;
  int G;                   // groups per row
  int log_group;           // 5, 6, 7
  int scale_bf16;
};

__device__ __forceinline__ uint32_t bf16_bits(float x) {  // to nearest, ties to even
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(0.f), "f"(x));
  return d & 0xffffu;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
constexpr int kInt4Threads = 256;
// place of a row's column among those that a warp's lanes exchange through shared memory: 16 to a lane, 17 apart
__device__ __forceinline__ int swap_at(int column) { return (column >> 4) * 17 + (column & 15); }

// ------------------------------------------------------------------------------------------
// Weights -> table.  A group's 32 .. 128 columns lie in 2 .. 8 neighbouring lanes, 16 columns each; the extremes meet
// by shuffles, so the weights are read once and nothing but the table is written.
// Roundings: the step to fp32 and to its type, the quotient weight / step to fp32, that to an integer
// (ties to even).  A group with a weight that is not finite gets the step NaN, codes and zero 0.
// The quotients are the reciprocal's product q corrected by its remainder, q + (x - q step) / step: three operations instead of a
// division each (128256 x 4096 bf16: 855 us with divisions).  Markstein's theorem gives the quotient rounded to nearest where
// q is off by less than a step of fp32, which in one pair of sixty it is not.  What is wanted are integers, and
// those hang on the quotients next to half steps: for every mantissa of the step and the five weights
// around each half step (671 million pairs, on the host) the corrected quotient is the division's.
// ------------------------------------------------------------------------------------------
struct QuantizeArgs {
  const void* w;
  long long stride;  // elements
  Int4Table T;
  int lanes;         // threads per row, a power of two
};

template <int DT, bool VEC>  // VEC: 16 columns of a row are aligned 16-byte words
__global__ void __launch_bounds__(kInt4Threads) quantize_kernel(const QuantizeArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4, kCols = 16;
  const Int4Table& T = A.T;
  const int per_group = 1 << (T.log_group - 4);  // lanes
  const int units = T.G * per_group, D = (int)T.D;
  const int at = threadIdx.x & (A.lanes - 1), rows = kInt4Threads / A.lanes;
  const int L = min(A.lanes, 32), l = threadIdx.x & (L - 1);  // lanes side by side in a row
  __shared__ float turns[VEC ? 1 : kInt4Threads * 17];
  float* const turn = turns + (VEC ? 0 : (threadIdx.x - l) * 17);
  const int bytes = (D + 1) >> 1;
  for (long long v0 = (long long)blockIdx.x * rows; v0 < T.V; v0 += (long long)gridDim.x * rows) {
    const long long v = v0 + threadIdx.x / A.lanes;
    const char* const row = (const char*)A.w + v * A.stride * ES;
    for (int first = 0; first < units; first += A.lanes) {  // the same number of rounds for every lane
      const int unit = first + at, d = unit * kCols;
      const bool live = v < T.V && unit < units;
      const int n = !live || d >= D ? 0 : min(D - d, kCols);
      float x[kCols];
      const char* p = row + (long long)d * ES;
      if (VEC && n == kCols) {
#pragma unroll
        for (int i = 0; i < kCols * ES / 16; ++i) {
          const uint4 q = ld_stream16(p + 16 * i);
          const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (DT == kBF16) x[8 * i + 2 * j] = bf16_lo(w[j]), x[8 * i + 2 * j + 1] = bf16_hi(w[j]);
            else x[4 * i + j] = __uint_as_float(w[j]);
          }
        }
      } else if (VEC) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          x[i] = 0.f;
          if (i < n)
            x[i] = DT == kBF16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)p + i) << 16) : __ldg((const float*)p + i);
        }
      } else {  // columns by neighbouring lanes, 16 each out of shared memory
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          const int col = (unit - l) * kCols + i * L + l;
          float y = 0.f;
          if (v < T.V && col < D)
            y = DT == kBF16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)row + col) << 16) : __ldg((const float*)row + col);
          turn[swap_at(i * L + l)] = y;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kCols; ++i) x[i] = turn[swap_at(l * kCols + i)];
      }
      float lo = 0.f, hi = 0.f, odd = 0.f;
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        odd = fmaf(x[i], 0.f, odd);  // NaN for infinities and NaN
        lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
      }
      for (int o = 1; o < per_group; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        odd += __shfl_xor_sync(0xffffffffu, odd, o);
      }
      const bool bad = odd != 0.f;
      float step = T.zeros ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(-lo, hi), 7.f);
      if (T.scale_bf16) step = __uint_as_float(bf16_bits(step) << 16);
      const bool some = step > 0.f && step <= 3.402823466e38f && !bad;
      const float zero = !T.zeros ? 8.f : some ? fminf(fmaxf(rintf(__fdiv_rn(-lo, step)), 0.f), 15.f) : 0.f;
      uint32_t word[2] = {0u, 0u};
      if (some && step >= 1e-30f) {
        const float inv = __frcp_rn(step), magic = 12582912.f;  // 1.5 * 2^23: integers in the lowest bits
        const int z = (int)zero - __float_as_int(magic);
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          const float q = x[i] * inv, r = fmaf(fmaf(-q, step, x[i]), inv, q);
          word[i >> 3] |= (uint32_t)__viaddmin_s32_relu(__float_as_int(r + magic), z, 15) << (4 * (i & 7));
        }
      } else if (some) {  // remainders that fp32 might not hold
        for (int i = 0; i < kCols; ++i) {
          const float q = fminf(fmaxf(rintf(__fdiv_rn(x[i], step)) + zero, 0.f), 15.f);
          if (i < 8) word[0] |= (uint32_t)q << (4 * i);
          else word[1] |= (uint32_t)q << (4 * (i - 8));
        }
      } else if (!bad) {
        word[0] = word[1] = (uint32_t)zero * 0x11111111u;
      }
      if (!live) continue;
      if (n < kCols) {
        const unsigned long long all = (unsigned long long)word[1] << 32 | word[0], some_of = all & ((1ull << (4 * n)) - 1ull);
        word[0] = (uint32_t)some_of, word[1] = (uint32_t)(some_of >> 32);
      }
      uint8_t* out = T.codes + v * T.code_stride + (d >> 1);
      if ((d >> 1) + 8 <= bytes) {
        *(uint2*)out = make_uint2(word[0], word[1]);
      } else {
        for (int i = 0; (d >> 1) + i < bytes; ++i) out[i] = (uint8_t)(word[i >> 2] >> (8 * (i & 3)));
      }
      if ((unit & (per_group - 1)) == 0) {
        const int g = unit >> (T.log_group - 4);
        const float s = bad || step > 3.402823466e38f ? __uint_as_float(0x7fc00000u) : step;
        if (T.scale_bf16) ((unsigned short*)T.scales)[v * T.scale_stride + g] = (unsigned short)(__float_as_uint(s) >> 16);
        else ((float*)T.scales)[v * T.scale_stride + g] = s;
        if (T.zeros) T.zeros[v * T.zero_stride + g] = (uint8_t)(bad ? 0.f : zero);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Rows by token, scaled: out[n,:] = scale * (step * (code - zero)), rounded to fp32 after each product and once to the
// output's type.  16 columns a thread; bound by the writes.  A code becomes a float without a conversion: 2^23 + code is
// its bits below an exponent, and the difference to 2^23 + zero is exact.
// ------------------------------------------------------------------------------------------
struct EmbedInt4Args {
  Int4Table T;
  const int32_t* tokens;
  long long N;
  float scale;
  char* out;
  long long out_stride;  // elements
  int lanes;             // threads per row, a power of two
  uint32_t* status;
};

template <int DT, bool VEC>  // VEC: 16 columns of a row of the output are aligned 16-byte words (of bf16)
__global__ void __launch_bounds__(kInt4Threads) embed_int4_kernel(const EmbedInt4Args A) {
  static_assert(!VEC || DT == kBF16, "fp32 rows go through shared memory");
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const Int4Table& T = A.T;
  const int units = (int)((T.D + 15) >> 4), D = (int)T.D;
  const int at = threadIdx.x & (A.lanes - 1), rows = kInt4Threads / A.lanes;
  const int L = min(A.lanes, 32), l = threadIdx.x & (L - 1);  // lanes side by side in a row
  __shared__ float turns[VEC ? 1 : kInt4Threads * 17];
  float* const turn = turns + (VEC ? 0 : (threadIdx.x - l) * 17);
  const long long step = (long long)gridDim.x * rows;
  long long n = (long long)blockIdx.x * rows + threadIdx.x / A.lanes;
  int next = n < A.N ? __ldg(A.tokens + n) : -1;
  for (long long n0 = (long long)blockIdx.x * rows; n0 < A.N; n0 += step, n += step) {  // the same for every lane
    const int t = next;
    if (n + step < A.N) next = __ldg(A.tokens + n + step);
    const bool row_there = n < A.N, live = row_there && t >= 0 && t < T.V;
    if (row_there && t >= T.V && at == 0 && A.status) atomicOr(A.status, 2u);
    const long long v = live ? t : 0;
    const uint8_t* const codes = T.codes + v * T.code_stride;
    const char* const scales = (const char*)T.scales + v * T.scale_stride * (T.scale_bf16 ? 2 : 4);
    const uint8_t* const zeros = T.zeros + (T.zeros ? v * T.zero_stride : 0);
    char* const row = A.out + n * A.out_stride * ES;
    for (int first = 0; first < units; first += A.lanes) {
      const int unit = first + at, d = unit * 16;
      float y[16];
      if (live && unit < units) {
        const uint2 w = __ldg((const uint2*)(codes + unit * 8));  // a row's codes fill 16-byte words
        const int g = unit >> (T.log_group - 4);
        const float s = T.scale_bf16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)scales + g) << 16) : __ldg((const float*)scales + g);
        const float z = __uint_as_float(0x4b000000u | (T.zeros ? (uint32_t)__ldg(zeros + g) & 15u : 8u));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t c = (i < 8 ? w.x : w.y) >> (4 * (i & 7));
          uint32_t bits;
          asm("lop3.b32 %0, %1, 0xf, 0x4b000000, 0xea;" : "=r"(bits) : "r"(c));
          y[i] = __fmul_rn(__uint_as_float(bits) - z, s);
        }
        if (A.scale != 1.f) {
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = __fmul_rn(y[i], A.scale);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
      }
      char* const q = row + (long long)d * ES;
      if (VEC) {
        if (!row_there || unit >= units) continue;
        if (d + 16 <= D) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            ((uint4*)q)[h] = make_uint4(bf16_pair(y[8 * h], y[8 * h + 1]), bf16_pair(y[8 * h + 2], y[8 * h + 3]),
                                        bf16_pair(y[8 * h + 4], y[8 * h + 5]), bf16_pair(y[8 * h + 6], y[8 * h + 7]));
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (d + i < D) ((unsigned short*)q)[i] = (unsigned short)bf16_bits(y[i]);
        }
      } else {  // out of shared memory, columns by neighbouring lanes
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) turn[swap_at(l * 16 + i)] = y[i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int col = (unit - l) * 16 + i * L + l;
          const float x = turn[swap_at(i * L + l)];
          if (row_there && col < D) {
            if constexpr (DT == kBF16) ((unsigned short*)row)[col] = (unsigned short)bf16_bits(x);
            else ((float*)row)[col] = x;
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Logits of hidden states: out[n,v] = sum_d x[n,d] * element(v, d).
//
// The product is mma.sync m16n8k16 with 16 table rows as the one operand and up to 8 hidden states as the other: for so
// few columns the codes' way into the registers, not the tensor pipe, is what costs, and there the operand comes straight
// from the lanes that converted it.  A code becomes bf16 without a conversion: 0x4300 | code is 128 + code, and
// (128 + code) - (128 + zero) is exact.  Which column of a sum goes to which k of an instruction is free as long as both
// operands agree, so a lane's 16 bytes (32 columns) feed the instructions in the order in which masks and
// shifts give them, and the hidden states lie in shared memory in that order.  A group's sum is multiplied by its
// scale in fp32.  fp32 hidden states are split into three bf16 parts (8 bits each, exactly), each with its own product.
//
// One or two hidden states (FEW): the instruction's eight columns are two hidden states times the four lanes of a
// quad: column 2 t + n holds hidden state n where the k belong to lane t and zeros elsewhere, so that the sums of
// lanes t come apart.  Each is of 32 neighbouring columns, hence of one group, whatever the groups' size, and lane t holds it.
// More: with groups of 128 a chunk of 128 columns has one scale per row; with smaller ones the lanes of
// a quad exchange their words first, so that an instruction's columns are of one group.
//
// A CTA has a range of tiles of 16 rows, cut into units of UC chunks of 128 columns; each warp takes a run of
// units of equal length, whatever the tiles, and streams them through a ring of its own: a tensor copy of 64 bytes of 16
// rows per chunk, which leaves what a warp reads at once side by side.  (Bulk copies row by row take one lane after
// the other: 262 instead of 150 instructions per chunk.)  The scales and zeros of a unit are requested when its codes are and stored
// beside them as pairs (fp32 scale, bf16 zero twice).  A tile that two or more warps share is added up at the end.
// ------------------------------------------------------------------------------------------
struct HeadArgs {
  Int4Table T;
  const char* x;
  long long x_stride;  // elements
  int N;
  char* out;
  long long out_stride;
  int out_bf16;
  int cols;            // hidden states per CTA row of the grid
  int chunks;          // of 128 columns
  int vec;             // a lane's scales and zeros of a unit are aligned vectors
  long long tiles;     // of 16 rows
};

constexpr int kHeadWarps = 16;  // at most: fewer where the hidden states leave no room for their rings
constexpr int kHeadStages = 2;

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Eight codes as bf16 differences to their zero, columns k and k + 4 as pairs.  Mask and magic in one instruction (written
// as & and | they are two: 22 instead of 14 integer instructions per two words).
__device__ __forceinline__ void int4_pairs(uint32_t w, uint32_t z, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t d;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(d) : "r"(w >> (4 * i)));
    p[i] = sub_bf16x2(d, z);
  }
}
// words of a quad's lanes exchanged: afterwards w[j] of lane t is what w[t] of lane j was
__device__ __forceinline__ void quad_transpose(uint32_t (&w)[4]) {
  const int t = threadIdx.x & 3;
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    const bool up = (t & o) != 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i & o) continue;
      const uint32_t send = up ? w[i] : w[i | o];
      const uint32_t got = __shfl_xor_sync(0xffffffffu, send, o);
      if (up) w[i] = got;
      else w[i | o] = got;
    }
  }
}
// the part of x that 8 bits hold (towards zero); the rest follows
__device__ __forceinline__ uint32_t take_bf16(float& x) {
  const uint32_t b = __float_as_uint(x);
  if ((b & 0x7f800000u) == 0x7f800000u) {  // infinities and NaN whole
    const uint32_t h = (b & 0x7fffffu) ? 0x7fc0u : b >> 16;
    x = 0.f;
    return h;
  }
  x = __fsub_rn(x, __uint_as_float(b & 0xffff0000u));
  return b >> 16;
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 b;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(at));
  return b;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 b;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(b.x), "=r"(b.y) : "r"(at));
  return b;
}

// A map's box, from column x of row y on; what lies outside comes as zeros
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t barrier) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to),
               "l"(map), "r"(x), "r"(y), "r"(barrier)
               : "memory");
}

template <int BYTES>
__device__ __forceinline__ void load_words(uint32_t* w, const char* p) {
  if constexpr (BYTES == 1) {
    w[0] = __ldg((const uint8_t*)p);
  } else if constexpr (BYTES == 2) {
    w[0] = __ldg((const unsigned short*)p);
  } else if constexpr (BYTES == 4) {
    w[0] = __ldg((const uint32_t*)p);
  } else if constexpr (BYTES == 8) {
    const uint2 q = __ldg((const uint2*)p);
    w[0] = q.x, w[1] = q.y;
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const uint4 q = __ldg((const uint4*)p + i);
      w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
    }
  }
}

// Shared memory of a head kernel: partial sums, per warp the ring and its barriers, zeros as far as a chunk of hidden
// states reaches, the hidden states.
struct HeadLayout {
  static constexpr int kRed = 2 * 128 * 4;  // per warp: two tiles of 8 columns
  static constexpr int kZeros = 2048;
  // a row's scales and zeros: rows of a warp's read in different banks (152064 x 4096, groups of 32: 211 us without)
  static __host__ __device__ constexpr int pitch(int gpc, int uc) { return gpc * uc * 8 + (gpc == 4 ? 32 : gpc == 2 ? 16 : 0); }
  static __host__ __device__ constexpr int stage(int gpc, int uc) { return 1024 * uc + 16 * pitch(gpc, uc); }
  static __host__ __device__ constexpr int fixed(int gpc, int uc, int warps) {
    return warps * (kRed + kHeadStages * (stage(gpc, uc) + 8)) + kZeros;
  }
};

// Groups' scales and zeros of a unit on their way: lane (row = lane / 2, half = lane % 2) has those of half a unit.
template <int GPC, int UC>
struct HeadScales {
  static constexpr int kMine = GPC * UC / 2;
  uint32_t scale[kMine], zero[(kMine + 3) / 4];

  __device__ __forceinline__ void load(const HeadArgs& A, long long v, int unit) {
    const Int4Table& T = A.T;
    const int g0 = unit * GPC * UC + (threadIdx.x & 1) * kMine;
    if (v >= T.V) v = T.V - 1;
    const char* s = (const char*)T.scales + (v * T.scale_stride + g0) * (T.scale_bf16 ? 2 : 4);
    if (A.vec && g0 + kMine <= T.G) {
      if (T.scale_bf16) load_words<kMine * 2>(scale, s);
      else load_words<kMine * 4>(scale, s);
      if (T.zeros) load_words<kMine>(zero, (const char*)T.zeros + v * T.zero_stride + g0);
    } else {
#pragma unroll
      for (int i = 0; i < (kMine + 3) / 4; ++i) zero[i] = 0u;
      if (T.scale_bf16) {
#pragma unroll
        for (int i = 0; i < (kMine + 1) / 2; ++i) scale[i] = 0u;
      }
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const bool in = g0 + i < T.G;
        if (T.scale_bf16) {
          if (in) scale[i >> 1] |= (uint32_t)__ldg((const unsigned short*)s + i) << (16 * (i & 1));
        } else {
          scale[i] = in ? __ldg((const uint32_t*)s + i) : 0u;
        }
        if (in && T.zeros) zero[i >> 2] |= (uint32_t)__ldg(T.zeros + v * T.zero_stride + g0 + i) << (8 * (i & 3));
      }
    }
  }
  // -> shared memory: [row][group of the unit] {fp32 scale, bf16 128 + zero twice}; the low four bits of a zero count
  __device__ __forceinline__ void store(const HeadArgs& A, uint32_t at) const {
    uint32_t out[2 * kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      out[2 * i] = !A.T.scale_bf16 ? scale[i] : i & 1 ? scale[i >> 1] & 0xffff0000u : scale[i >> 1] << 16;
      const uint32_t z = A.T.zeros ? zero[i >> 2] & 0x0f0f0f0fu : 0x08080808u;
      out[2 * i + 1] = __byte_perm(z, 0x43u, 0x4040u | (uint32_t)(i & 3) * 0x0101u);
    }
    at += threadIdx.x % 32 / 2 * HeadLayout::pitch(GPC, UC) + (threadIdx.x & 1) * (kMine * 8);
    if constexpr (kMine == 1) {
      asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(out[0]), "r"(out[1]) : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < kMine / 2; ++i)
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at + 16 * i), "r"(out[4 * i]), "r"(out[4 * i + 1]),
                     "r"(out[4 * i + 2]), "r"(out[4 * i + 3])
                     : "memory");
    }
  }
};

// FEW: 1 or 2, the hidden states at most; 0: up to 8
template <int GPC, int PARTS, int FEW, int UC>
__global__ void __launch_bounds__(32 * kHeadWarps, 1) head_kernel(const HeadArgs A, const __grid_constant__ CUtensorMap codes) {
  extern __shared__ __align__(1024) char head_shared[];
  constexpr bool kQuad = FEW || GPC == 1;  // a lane's words stay its own
  constexpr int kStage = HeadLayout::stage(GPC, UC);
  const Int4Table& T = A.T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int n0 = blockIdx.y * A.cols, cols = min(A.cols, A.N - n0);
  const int width = FEW ? FEW : cols;  // columns that the hidden states' layout has
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(head_shared);
  const int warps = blockDim.x >> 5;
  float* const red = (float*)head_shared;  // [warp][2][8][16]
  const uint32_t ring = base + warps * HeadLayout::kRed + warp * (kHeadStages * kStage);
  const int bars_at = warps * (HeadLayout::kRed + kHeadStages * kStage), zeros_at = bars_at + warps * kHeadStages * 8;
  const uint32_t bars = base + bars_at + warp * (kHeadStages * 8);
  const int chunks_up = (A.chunks + UC - 1) / UC * UC;
  const int plane = chunks_up * 16 * width;  // 16-byte units per part

  const long long units_per_row = (A.chunks + UC - 1) / UC;
  const long long t0 = A.tiles * blockIdx.x / gridDim.x, t1 = A.tiles * (blockIdx.x + 1) / gridDim.x;
  const long long all = (t1 - t0) * units_per_row;
  const int first = (int)(all * warp / warps), last = (int)(all * (warp + 1) / warps);
  const int upr = (int)units_per_row;

  // requests run kHeadStages units ahead of the products
  long long l_tile = t0 + first / upr;
  int l_unit = first % upr;
  HeadScales<GPC, UC> scales[kHeadStages];
  auto request = [&](int stage) {
    const uint32_t bar = bars + stage * 8;
    if (elected()) {
      barrier_expect(bar, UC * 1024);
#pragma unroll
      for (int c = 0; c < UC; ++c)
        copy_box(ring + stage * kStage + c * 1024, &codes, (l_unit * UC + c) * 64, (int)(l_tile * 16), bar);
    }
    scales[stage].load(A, l_tile * 16 + (lane >> 1), l_unit);
    if (++l_unit == upr) l_unit = 0, ++l_tile;
  };
  if (lane < kHeadStages) barrier_init(bars + lane * 8, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
#pragma unroll
  for (int q = 0; q < kHeadStages; ++q)
    if (first + q < last) request(q);

  // hidden states -> shared memory in parts of bf16: unit (chunk, j, n, t) holds 8 columns as pairs (k, k + 4), of a lane's
  // own 32 columns, or of those that a quad's lanes have after exchanging their words
  uint4* const xs = (uint4*)(head_shared + zeros_at);
  for (int i = threadIdx.x; i < HeadLayout::kZeros / 16; i += blockDim.x) xs[i] = make_uint4(0u, 0u, 0u, 0u);
  for (int i = threadIdx.x; i < plane; i += blockDim.x) {
    const int t = i & 3, n = (i >> 2) % width, cj = (i >> 2) / width, j = cj & 3, c = cj >> 2;
    const long long d = (long long)c * 128 + (kQuad ? t * 32 + j * 8 : j * 32 + t * 8);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.f;
      if (d + e < T.D && n < cols) {
        const long long at = (long long)(n0 + n) * A.x_stride + d + e;
        v[e] = PARTS == 1 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)A.x + at) << 16) : __ldg((const float*)A.x + at);
      }
    }
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = PARTS == 1 ? __float_as_uint(v[e]) >> 16 : take_bf16(v[e]);
      xs[HeadLayout::kZeros / 16 + (size_t)part * plane + i] = make_uint4(h[0] | h[4] << 16, h[1] | h[5] << 16, h[2] | h[6] << 16, h[3] | h[7] << 16);
    }
  }
  __syncthreads();

  // where the hidden states of the lane's columns lie, bytes from one chunk to the next and from one part to the next;
  // lanes without one read zeros
  const uint32_t x_j = (uint32_t)width * 64u;
  const bool there = FEW ? tig == gid >> 1 && (gid & 1) < FEW : gid < cols;
  const uint32_t x_at = base + zeros_at + (there ? HeadLayout::kZeros + ((FEW ? gid & 1 : gid) * 4 + tig) * 16 : 0);
  const uint32_t x_chunk = there ? 4u * x_j : 0u, x_part = there ? (uint32_t)plane * 16u : 0u;

  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  auto put = [&](int i, long long tile, float y) {
    const long long v = tile * 16 + (i & 15);
    if (v >= T.V) return;
    const long long at = (long long)(n0 + (i >> 4)) * A.out_stride + v;
    if (A.out_bf16) ((unsigned short*)A.out)[at] = (unsigned short)bf16_bits(y);
    else ((float*)A.out)[at] = y;
  };
  long long tile = t0 + first / upr;
  int unit = first % upr, phase = 0;
  bool whole = unit == 0, lost = false;  // whole: all of the tile so far is this warp's
  for (int u0 = first; u0 < last; u0 += kHeadStages, phase ^= 1) {
#pragma unroll
    for (int q = 0; q < kHeadStages; ++q) {
      if (u0 + q >= last) break;
      const uint32_t stage_at = ring + q * kStage, scale_at = stage_at + UC * 1024;
      scales[q].store(A, scale_at);
      lost |= !barrier_wait(bars + q * 8, phase);
      __syncwarp();
      const uint32_t code_at = stage_at + lane * 16;
      const uint32_t sc_at = scale_at + gid * HeadLayout::pitch(GPC, UC) + (FEW ? tig * GPC >> 2 : 0) * 8;
      uint32_t xa = x_at + (uint32_t)(unit * UC) * x_chunk;
#pragma unroll
      for (int c = 0; c < UC; ++c) {
        const uint4 c0 = lds16(code_at + c * 1024), c1 = lds16(code_at + c * 1024 + 512);
        uint32_t w[2][4] = {{c0.x, c0.y, c0.z, c0.w}, {c1.x, c1.y, c1.z, c1.w}};
        if (!kQuad) quad_transpose(w[0]), quad_transpose(w[1]);
        constexpr int kSets = FEW ? 1 : GPC;  // sums of one scale each
#pragma unroll
        for (int g = 0; g < kSets; ++g) {
          const uint2 s0 = lds8(sc_at + (c * GPC + g) * 8), s1 = lds8(sc_at + 8 * HeadLayout::pitch(GPC, UC) + (c * GPC + g) * 8);
          float sum[2][4];  // two chains of products
#pragma unroll
          for (int jj = 0; jj < 4 / kSets; ++jj) {
            const int j = g * (4 / kSets) + jj;
            uint32_t p0[4], p1[4];
            int4_pairs(w[0][j], s0.y, p0);
            int4_pairs(w[1][j], s1.y, p1);
            const uint32_t a0[4] = {p0[0], p1[0], p0[1], p1[1]}, a1[4] = {p0[2], p1[2], p0[3], p1[3]};
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const uint4 b = lds16(xa + (uint32_t)j * x_j + (uint32_t)part * x_part);
              if (jj == 0 && part == 0) {
                mma_bf16_first(sum[0], a0, b.x, b.y);
                mma_bf16_first(sum[1], a1, b.z, b.w);
              } else {
                mma_bf16(sum[0], a0, b.x, b.y);
                mma_bf16(sum[1], a1, b.z, b.w);
              }
            }
          }
          const float f0 = __uint_as_float(s0.x), f1 = __uint_as_float(s1.x);
          acc[0] += f0 * (sum[0][0] + sum[1][0]);
          acc[1] += f0 * (sum[0][1] + sum[1][1]);
          acc[2] += f1 * (sum[0][2] + sum[1][2]);
          acc[3] += f1 * (sum[0][3] + sum[1][3]);
        }
        xa += x_chunk;
      }
      __syncwarp();  // the stage has been read
      if (u0 + q + kHeadStages < last) request(q);
      const bool row_end = ++unit == upr;
      if (row_end || u0 + q + 1 == last) {
        // the sums of the tile, or of the warp's part of it: [column][row].  The first slot keeps the end of a tile that
        // an earlier warp began, the second one whole tiles on their way and at last a part without the tile's end.
        float* const slot = red + (warp * 2 + (row_end && !whole ? 0 : 1)) * 128;
        if (FEW) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 1);
            acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 2);
          }
        }
        const float bad = lost ? __uint_as_float(0x7fc00000u) : 0.f;
        if (!FEW || tig == 0) {
          float* at = slot + (FEW ? 0 : 2 * tig) * 16 + gid;
          at[0] = acc[0] + bad, at[16] = acc[1] + bad, at[8] = acc[2] + bad, at[24] = acc[3] + bad;
        }
        acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
        if (row_end && whole) {
          __syncwarp();
          for (int i = lane; i < 16 * cols; i += 32) put(i, tile, slot[i]);
          __syncwarp();
        }
        if (row_end) unit = 0, whole = true, ++tile;
      }
    }
  }
  __syncthreads();
  // a tile that this warp began and others went on with: parts in order
  const int begun = last / upr * upr, end = begun + upr;
  if (first < last && last % upr != 0 && begun >= first) {
    int parts = warp + 1;  // warps up to the one that has the tile's end
    while ((int)(all * (parts + 1) / warps) < end) ++parts;
    for (int i = lane; i < 16 * cols; i += 32) {
      float y = red[(warp * 2 + 1) * 128 + i];
      for (int w = warp + 1; w <= parts; ++w)
        if (all * w / warps < all * (w + 1) / warps) y += red[(w * 2 + (w < parts ? 1 : 0)) * 128 + i];
      put(i, t0 + last / upr, y);
    }
  }
}

}  // namespace gls
