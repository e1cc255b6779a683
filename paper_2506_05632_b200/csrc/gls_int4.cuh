// gls_int4.cuh -- a table of V rows of D columns at 4 bits with a step (and a zero) per group of columns:
//     element (v, d) = scale[v, d / group] * (code[v, d] - zero[v, d / group])      zero 8 where none are given
// made from weights, read back by token, and multiplied with hidden states (the logits of a 4-bit head).
// Two codes a byte, the even column in the low half; a row's codes start on a 16-byte boundary.
#pragma once
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
__device__ __forceinline__ float int4_scale(const Int4Table& T, long long v, int g) {
  const long long i = v * T.scale_stride + g;
  return T.scale_bf16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)T.scales + i) << 16)
                      : __ldg((const float*)T.scales + i);
}
__device__ __forceinline__ uint32_t int4_zero(const Int4Table& T, long long v, int g) {
  return T.zeros ? (uint32_t)__ldg(T.zeros + v * T.zero_stride + g) & 15u : 8u;
}

constexpr int kInt4Threads = 256;

// ------------------------------------------------------------------------------------------
// Weights -> table.  A group's 32 .. 128 columns lie in 4 .. 16 neighbouring lanes, 8 columns each; the extremes meet
// by shuffles, so the weights are read once and nothing but the table is written (bound by HBM).
// Roundings: the step to fp32 and to its type, the quotient weight / step to fp32, that to an integer
// (ties to even).  A group with a weight that is not finite gets the step NaN, codes and zero 0.
// ------------------------------------------------------------------------------------------
struct QuantizeArgs {
  const void* w;
  long long stride;  // elements
  Int4Table T;
  int vec;           // 1: 8 columns of a row are aligned 16-byte words
  int lanes;         // threads per row, a power of two
};

template <int DT>
__global__ void __launch_bounds__(kInt4Threads) quantize_kernel(const QuantizeArgs A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const Int4Table& T = A.T;
  const int per_group = 1 << (T.log_group - 3);  // lanes
  const int units = T.G * per_group;
  const int at = threadIdx.x & (A.lanes - 1), rows = kInt4Threads / A.lanes;
  const long long bytes = (T.D + 1) >> 1;
  for (long long v0 = (long long)blockIdx.x * rows; v0 < T.V; v0 += (long long)gridDim.x * rows) {
    const long long v = v0 + threadIdx.x / A.lanes;
    for (int base = 0; base < units; base += A.lanes) {  // the same number of rounds for every lane
      const int unit = base + at;
      const bool live = v < T.V && unit < units;
      const long long d = (long long)unit * 8;
      const int n = !live || d >= T.D ? 0 : T.D - d < 8 ? (int)(T.D - d) : 8;
      float x[8];
      const char* p = (const char*)A.w + (v * A.stride + d) * ES;
      if (A.vec && n == 8) {
        if constexpr (DT == kBF16) {
          const uint4 q = ld_stream16(p);
          const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 q = ld_stream16(p + 16 * i);
            x[4 * i] = __uint_as_float(q.x), x[4 * i + 1] = __uint_as_float(q.y);
            x[4 * i + 2] = __uint_as_float(q.z), x[4 * i + 3] = __uint_as_float(q.w);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = 0.f;
          if (i < n)
            x[i] = DT == kBF16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)p + i) << 16) : __ldg((const float*)p + i);
        }
      }
      float lo = 0.f, hi = 0.f;
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bad |= !(fabsf(x[i]) <= 3.402823466e38f);
        lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
      }
      for (int o = 1; o < per_group; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
      }
      float step = T.zeros ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(-lo, hi), 7.f);
      const uint32_t step16 = bf16_bits(step);
      if (T.scale_bf16) step = __uint_as_float(step16 << 16);
      const bool some = step > 0.f && step <= 3.402823466e38f && !bad;
      const float zero = !T.zeros ? 8.f : some ? fminf(fmaxf(rintf(__fdiv_rn(-lo, step)), 0.f), 15.f) : 0.f;
      uint32_t word = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float q = zero;
        if (some) q = fminf(fmaxf(rintf(__fdiv_rn(x[i], step)) + zero, 0.f), 15.f);
        if (bad) q = 0.f;
        word |= (i < n ? (uint32_t)q : 0u) << (4 * i);
      }
      if (!live) continue;
      uint8_t* out = T.codes + v * T.code_stride + (d >> 1);
      if ((d >> 1) + 4 <= bytes) {
        *(uint32_t*)out = word;
      } else {
        for (int i = 0; (d >> 1) + i < bytes; ++i) out[i] = (uint8_t)(word >> (8 * i));
      }
      if ((unit & (per_group - 1)) == 0) {
        const int g = unit >> (T.log_group - 3);
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
// output's type.  8 columns a thread; bound by the writes.
// ------------------------------------------------------------------------------------------
struct EmbedInt4Args {
  Int4Table T;
  const int32_t* tokens;
  long long N;
  float scale;
  char* out;
  long long out_stride;  // elements
  int vec, lanes;
  uint32_t* status;
};

template <int DT>
__global__ void __launch_bounds__(kInt4Threads) embed_int4_kernel(const EmbedInt4Args A) {
  constexpr int ES = DT == kBF16 ? 2 : 4;
  const Int4Table& T = A.T;
  const int units = (int)((T.D + 7) >> 3);
  const int at = threadIdx.x & (A.lanes - 1), rows = kInt4Threads / A.lanes;
  const long long bytes = (T.D + 1) >> 1;
  for (long long n0 = (long long)blockIdx.x * rows; n0 < A.N; n0 += (long long)gridDim.x * rows) {
    const long long n = n0 + threadIdx.x / A.lanes;
    if (n >= A.N) continue;
    const int t = __ldg(A.tokens + n);
    const bool live = t >= 0 && t < T.V;
    if (t >= T.V && at == 0 && A.status) atomicOr(A.status, 2u);
    for (int unit = at; unit < units; unit += A.lanes) {
      const long long d = (long long)unit * 8;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = 0.f;
      if (live) {
        const uint8_t* p = T.codes + t * T.code_stride + (d >> 1);
        uint32_t word = 0u;
        if ((d >> 1) + 4 <= bytes) {
          word = __ldg((const uint32_t*)p);
        } else {
          for (int i = 0; (d >> 1) + i < bytes; ++i) word |= (uint32_t)__ldg(p + i) << (8 * i);
        }
        const int g = unit >> (T.log_group - 3);
        const float s = int4_scale(T, t, g), z = (float)int4_zero(T, t, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(__fmul_rn((float)((word >> (4 * i)) & 15u) - z, s), A.scale);
      }
      char* q = A.out + (n * A.out_stride + d) * ES;
      if (A.vec && d + 8 <= T.D) {
        if constexpr (DT == kBF16) {
          *(uint4*)q = make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7]));
        } else {
          ((float4*)q)[0] = make_float4(y[0], y[1], y[2], y[3]);
          ((float4*)q)[1] = make_float4(y[4], y[5], y[6], y[7]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (d + i < T.D) {
            if constexpr (DT == kBF16) ((unsigned short*)q)[i] = (unsigned short)bf16_bits(y[i]);
            else ((float*)q)[i] = y[i];
          }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Logits of hidden states: out[n,v] = sum_d x[n,d] * element(v, d).
//
// The product is mma.sync m16n8k16 with 16 table rows as the one operand and up to 8 hidden states as the other: for so
// few columns the codes' way into the registers, not the tensor pipe, is what costs, and there A comes straight from the
// lanes that loaded and converted it.  A code becomes bf16 without a conversion: 0x4300 | code is 128 + code, and
// (128 + code) - (128 + zero) is exact.  Which column of a sum goes to which k of an instruction is free as long as both
// operands agree, so a lane's 16 loaded bytes (32 columns) feed the instructions in the order in which masks and
// shifts give them, and the hidden states lie in shared memory in that order.  With groups of 128
// a chunk of 128 columns has one step per row; with smaller groups the lanes of a quad exchange their words, so that an
// instruction's columns are of one group.  A group's sum is multiplied by its step in fp32.
// fp32 hidden states are split into three bf16 parts (8 bits each, exactly), each with its own product.
//
// A team of warps takes 16 rows, a warp every team-th chunk of 128 columns (1 KB of codes, the next three already
// requested); the team's sums meet in shared memory.
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
  int team;            // warps per 16 rows: 1, 2, 4, 8, 16
  int chunks;          // of 128 columns
  long long tiles;     // of 16 rows
};

constexpr int kHeadThreads = 512;

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
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

__device__ __forceinline__ void team_sync(int team, int threads) {  // barrier 0 is the whole CTA's
  if (threads == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(threads) : "memory");
}

// How the scales come: as one aligned vector per row and step of that type, or one by one.
enum : int { kScalesF32 = 0, kScalesBF16 = 1, kScalesAny = 2 };

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

// A step: 256 columns of 16 rows.  Lane (gid, tig) has columns 32 tig .. 32 tig + 31 of each half for rows gid, gid + 8.
template <int GPC, int ST>  // groups per 128 columns
struct HeadStep {
  static constexpr int kGroups = 2 * GPC;
  static constexpr int kWords = ST == kScalesBF16 ? GPC : kGroups;  // raw scales per row
  uint4 code[2][2];  // [row][half]
  uint32_t scale[2][kWords];
  uint32_t zero[2][(kGroups + 3) / 4];  // a byte per group
  __device__ __forceinline__ float step(int r, int g) const {
    if constexpr (ST == kScalesBF16) return __uint_as_float(g & 1 ? scale[r][g >> 1] & 0xffff0000u : scale[r][g >> 1] << 16);
    else return __uint_as_float(scale[r][g]);
  }
  // 128 + zero twice, in bf16; the low four bits of a zero count
  __device__ __forceinline__ uint32_t zero_pair(int r, int g) const {
    return __byte_perm(zero[r][g >> 2] & 0x0f0f0f0fu, 0x43u, 0x4040u | (uint32_t)(g & 3) * 0x0101u);
  }
};

// Position of a warp in its CTA's share of the table: teams of warps take tiles of 16 rows, a warp every team-th step of
// them, and its requests run some steps ahead of its products, across tiles.
struct HeadWalk {
  int in_team, team, rounds, steps_per_row;
  long long first, stride;
  int steps;
  __device__ __forceinline__ HeadWalk(const HeadArgs& A, int teams, int my_team, int warp_in_team) {
    in_team = warp_in_team;
    team = A.team;
    steps_per_row = (A.chunks + 1) >> 1;
    rounds = (steps_per_row + team - 1) / team;
    first = (long long)blockIdx.x * teams + my_team;
    stride = (long long)gridDim.x * teams;
    steps = (int)(first < A.tiles ? (A.tiles - first + stride - 1) / stride : 0) * rounds;
  }
};

// A 4-column pair of codes as bf16 differences to their zero
__device__ __forceinline__ void int4_pairs(uint32_t w, uint32_t z, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = sub_bf16x2(((w >> (4 * i)) & 0x000f000fu) | 0x43004300u, z);
}

__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 b;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(at));
  return b;
}

// Hidden states -> shared memory in parts of bf16: unit (chunk, j, n, t) holds 8 columns as pairs (k, k + 4); QUAD: those
// of a lane's own 32 columns, otherwise those that the exchanged words of a quad are of.
template <int PARTS, bool QUAD>
__device__ __forceinline__ void stage_hidden(const HeadArgs& A, uint4* xs, int n0, int cols, int units, int plane) {
  for (int i = threadIdx.x; i < units; i += kHeadThreads) {
    const int t = i & 3, n = (i >> 2) % cols, cj = (i >> 2) / cols, j = cj & 3, c = cj >> 2;
    const long long d = (long long)c * 128 + (QUAD ? t * 32 + j * 8 : j * 32 + t * 8);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.f;
      if (d + e < A.T.D) {
        const long long at = (long long)(n0 + n) * A.x_stride + d + e;
        v[e] = PARTS == 1 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)A.x + at) << 16) : __ldg((const float*)A.x + at);
      }
    }
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = PARTS == 1 ? __float_as_uint(v[e]) >> 16 : take_bf16(v[e]);
      xs[(size_t)part * plane + i] = make_uint4(h[0] | h[4] << 16, h[1] | h[5] << 16, h[2] | h[6] << 16, h[3] | h[7] << 16);
    }
  }
}

// The sums that a team's warps left in `red` [warp][column][row], added up and stored.
template <int NT>
__device__ __forceinline__ void head_store(const HeadArgs& A, const float* team_at, int thread, int threads, int n0, int cols, long long tile) {
  for (int i = thread; i < 16 * cols; i += threads) {
    float y = 0.f;
    for (int k = 0; k < A.team; ++k) y += team_at[k * 128 * NT + i];
    const long long v = tile * 16 + (i & 15);
    if (v < A.T.V) {
      const long long at = (long long)(n0 + (i >> 4)) * A.out_stride + v;
      if (A.out_bf16) ((unsigned short*)A.out)[at] = (unsigned short)bf16_bits(y);
      else ((float*)A.out)[at] = y;
    }
  }
}

template <int GPC, int PARTS, int NT, int ST>
__global__ void __launch_bounds__(kHeadThreads, 1) head_kernel(const HeadArgs A) {
  extern __shared__ __align__(16) uint4 head_shared[];
  typedef HeadStep<GPC, ST> Step;
  constexpr int kAhead = GPC == 4 || (GPC == 2 && ST != kScalesBF16) ? 1 : 2;  // what registers hold
  const Int4Table& T = A.T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int n0 = blockIdx.y * A.cols, cols = min(A.cols, A.N - n0);
  const int chunks2 = (A.chunks + 1) & ~1;
  const int plane = chunks2 * 16 * cols;      // 16-byte units per part
  float* const red = (float*)head_shared;     // [16 warps][8 NT][16]
  uint4* const xs = head_shared + 16 * 32 * NT;  // a unit of zeros, then the hidden states
  if (threadIdx.x == 0) xs[0] = make_uint4(0u, 0u, 0u, 0u);
  stage_hidden<PARTS, GPC == 1>(A, xs + 1, n0, cols, plane, plane);
  __syncthreads();

  const int teams = kHeadThreads / 32 / A.team, my_team = warp / A.team;
  const HeadWalk W(A, teams, my_team, warp % A.team);
  const int row_last = (int)((T.D + 31) / 32 * 16) - 16;

  // What the next request reads: step l_step of the rows at l_code.  Codes and scales behind a row's end
  // are replaced by its last ones: the hidden states there are zeros.
  long long l_tile = W.first;
  int l_step = W.in_team;
  const uint8_t* l_code[2];
  const char* l_scale[2];
  const uint8_t* l_zero[2];
  constexpr int ss = ST == kScalesBF16 ? 2 : 4;
  const int ss_any = T.scale_bf16 ? 2 : 4;
  auto aim = [&]() {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      long long v = l_tile * 16 + gid + 8 * r;
      if (v >= T.V) v = T.V - 1;  // read again, not stored
      l_code[r] = T.codes + v * T.code_stride;
      l_scale[r] = (const char*)T.scales + v * T.scale_stride * (ST == kScalesAny ? ss_any : ss);
      l_zero[r] = T.zeros + v * T.zero_stride;
    }
  };
  aim();
  auto request = [&](Step& h) {
    const int at0 = min(l_step * 128 + tig * 16, row_last), at1 = min(l_step * 128 + tig * 16 + 64, row_last);
    const int s = min(l_step, W.steps_per_row - 1);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      h.code[r][0] = ld_stream16(l_code[r] + at0);
      h.code[r][1] = ld_stream16(l_code[r] + at1);
      if constexpr (ST == kScalesAny) {
#pragma unroll
        for (int g = 0; g < Step::kGroups; ++g) {
          const int gg = min(s * Step::kGroups + g, T.G - 1);
          h.scale[r][g] = T.scale_bf16 ? (uint32_t)__ldg((const unsigned short*)l_scale[r] + gg) << 16 : __ldg((const uint32_t*)l_scale[r] + gg);
        }
      } else {
        load_words<Step::kGroups * ss>(h.scale[r], l_scale[r] + s * (Step::kGroups * ss));
      }
      if (T.zeros) {
        if constexpr (ST == kScalesAny) {
#pragma unroll
          for (int i = 0; i < (Step::kGroups + 3) / 4; ++i) h.zero[r][i] = 0u;
#pragma unroll
          for (int g = 0; g < Step::kGroups; ++g)
            h.zero[r][g >> 2] |= (uint32_t)__ldg(l_zero[r] + min(s * Step::kGroups + g, T.G - 1)) << (8 * (g & 3));
        } else {
          load_words<Step::kGroups>(h.zero[r], (const char*)l_zero[r] + s * Step::kGroups);
        }
      } else {
#pragma unroll
        for (int i = 0; i < (Step::kGroups + 3) / 4; ++i) h.zero[r][i] = 0x08080808u;
      }
    }
    l_step += W.team;
    if (l_step >= W.rounds * W.team) {
      l_step = W.in_team;
      l_tile += W.stride;
      aim();
    }
  };

  // where the hidden states of the lane's columns lie: bytes, and from one j to the next
  uint32_t x_at[NT], x_step[NT], x_part[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const bool there = gid + 8 * nt < cols;
    x_at[nt] = (uint32_t)__cvta_generic_to_shared(xs) + (there ? 16u + ((gid + 8 * nt) * 4 + tig) * 16u : 0u);
    x_step[nt] = there ? (uint32_t)cols * 64u : 0u;
    x_part[nt] = there ? (uint32_t)plane * 16u : 0u;
  }

  Step ring[kAhead];
#pragma unroll
  for (int q = 0; q < kAhead; ++q)
    if (q < W.steps) request(ring[q]);
  float acc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
  long long tile = W.first;
  int s = W.in_team;
  for (int s0 = 0; s0 < W.steps; s0 += kAhead) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (s0 + q >= W.steps) break;
      Step& h = ring[q];
      if (s < W.steps_per_row) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t w[2][4];
#pragma unroll
          for (int r = 0; r < 2; ++r) w[r][0] = h.code[r][half].x, w[r][1] = h.code[r][half].y, w[r][2] = h.code[r][half].z, w[r][3] = h.code[r][half].w;
          if (GPC > 1) quad_transpose(w[0]), quad_transpose(w[1]);
          uint32_t xa[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) xa[nt] = x_at[nt] + (uint32_t)(2 * s + half) * 4u * x_step[nt];
#pragma unroll
          for (int gl = 0; gl < GPC; ++gl) {
            const int g = half * GPC + gl;
            float sum[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sum[nt][0] = sum[nt][1] = sum[nt][2] = sum[nt][3] = 0.f;
            const uint32_t z0 = h.zero_pair(0, g), z1 = h.zero_pair(1, g);
#pragma unroll
            for (int jj = 0; jj < 4 / GPC; ++jj) {
              const int j = gl * (4 / GPC) + jj;
              uint32_t p0[4], p1[4];
              int4_pairs(w[0][j], z0, p0);
              int4_pairs(w[1][j], z1, p1);
              const uint32_t a0[4] = {p0[0], p1[0], p0[1], p1[1]}, a1[4] = {p0[2], p1[2], p0[3], p1[3]};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                  const uint4 b = lds16(xa[nt] + (uint32_t)part * x_part[nt]);
                  mma_bf16(sum[nt], a0, b.x, b.y);
                  mma_bf16(sum[nt], a1, b.z, b.w);
                }
                xa[nt] += x_step[nt];
              }
            }
            const float s0v = h.step(0, g), s1v = h.step(1, g);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              acc[nt][0] += s0v * sum[nt][0];
              acc[nt][1] += s0v * sum[nt][1];
              acc[nt][2] += s1v * sum[nt][2];
              acc[nt][3] += s1v * sum[nt][3];
            }
          }
        }
      }
      if (s0 + q + kAhead < W.steps) request(h);
      s += W.team;
      if (s >= W.rounds * W.team) {
        float* q_at = red + warp * 128 * NT + 2 * tig * 16 + gid;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          q_at[128 * nt] = acc[nt][0], q_at[128 * nt + 16] = acc[nt][1];
          q_at[128 * nt + 8] = acc[nt][2], q_at[128 * nt + 24] = acc[nt][3];
          acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
        }
        team_sync(my_team, W.team * 32);
        head_store<NT>(A, red + my_team * W.team * 128 * NT, W.in_team * 32 + lane, W.team * 32, n0, cols, tile);
        team_sync(my_team, W.team * 32);
        s = W.in_team;
        tile += W.stride;
      }
    }
  }
}

// The same for one or two hidden states.  The instruction's eight columns then are two hidden states times the four
// lanes of a quad: column 2 t + n holds hidden state n where the k belong to lane t and zeros elsewhere, so that the sums of
// lanes t come apart.  Each is of 32 neighbouring columns, hence of one group, whatever the groups' size, and lane t
// holds it: it multiplies it by its own scale, no words are exchanged, and scales need no alignment.
template <int PARTS, int ST>
__global__ void __launch_bounds__(kHeadThreads, 1) head_few_kernel(const HeadArgs A) {
  extern __shared__ __align__(16) uint4 head_shared[];
  constexpr int kAhead = 2;
  const Int4Table& T = A.T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int n0 = blockIdx.y * A.cols, cols = min(A.cols, A.N - n0);
  const int chunks2 = (A.chunks + 1) & ~1;
  const int plane = chunks2 * 16 * cols;
  float* const red = (float*)head_shared;
  uint4* const xs = head_shared + 16 * 32;
  if (threadIdx.x == 0) xs[0] = make_uint4(0u, 0u, 0u, 0u);
  stage_hidden<PARTS, true>(A, xs + 1, n0, cols, plane, plane);
  __syncthreads();

  const int teams = kHeadThreads / 32 / A.team, my_team = warp / A.team;
  const HeadWalk W(A, teams, my_team, warp % A.team);
  const int row_last = (int)((T.D + 31) / 32 * 16) - 16;
  struct Step {
    uint4 code[2][2];
    uint32_t scale[2][2], zero[2][2];
  };
  long long l_tile = W.first;
  int l_step = W.in_team;
  const uint8_t* l_code[2];
  const char* l_scale[2];
  const uint8_t* l_zero[2];
  constexpr int ss = ST == kScalesBF16 ? 2 : 4;
  auto aim = [&]() {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      long long v = l_tile * 16 + gid + 8 * r;
      if (v >= T.V) v = T.V - 1;
      l_code[r] = T.codes + v * T.code_stride;
      l_scale[r] = (const char*)T.scales + v * T.scale_stride * ss;
      l_zero[r] = T.zeros + v * T.zero_stride;
    }
  };
  aim();
  auto request = [&](Step& h) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = min(l_step * 128 + half * 64 + tig * 16, row_last), g = at >> (T.log_group - 1);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        h.code[r][half] = ld_stream16(l_code[r] + at);
        load_words<ss>(&h.scale[r][half], l_scale[r] + g * ss);
        h.zero[r][half] = 8u;
        if (T.zeros) h.zero[r][half] = __ldg(l_zero[r] + g);
      }
    }
    l_step += W.team;
    if (l_step >= W.rounds * W.team) {
      l_step = W.in_team;
      l_tile += W.stride;
      aim();
    }
  };
  const bool there = tig == gid >> 1 && (gid & 1) < cols;
  const uint32_t x_at = (uint32_t)__cvta_generic_to_shared(xs) + (there ? 16u + ((gid & 1) * 4 + tig) * 16u : 0u);
  const uint32_t x_step = there ? (uint32_t)cols * 64u : 0u, x_part = there ? (uint32_t)plane * 16u : 0u;

  Step ring[kAhead];
#pragma unroll
  for (int q = 0; q < kAhead; ++q)
    if (q < W.steps) request(ring[q]);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  long long tile = W.first;
  int s = W.in_team;
  for (int s0 = 0; s0 < W.steps; s0 += kAhead) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (s0 + q >= W.steps) break;
      Step& h = ring[q];
      if (s < W.steps_per_row) {
        uint32_t xa = x_at + (uint32_t)s * 8u * x_step;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t w[2][4] = {{h.code[0][half].x, h.code[0][half].y, h.code[0][half].z, h.code[0][half].w},
                                    {h.code[1][half].x, h.code[1][half].y, h.code[1][half].z, h.code[1][half].w}};
          const uint32_t z0 = ((h.zero[0][half] & 15u) | 0x4300u) * 0x10001u, z1 = ((h.zero[1][half] & 15u) | 0x4300u) * 0x10001u;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t p0[4], p1[4];
            int4_pairs(w[0][j], z0, p0);
            int4_pairs(w[1][j], z1, p1);
            const uint32_t a0[4] = {p0[0], p1[0], p0[1], p1[1]}, a1[4] = {p0[2], p1[2], p0[3], p1[3]};
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const uint4 b = lds16(xa + (uint32_t)part * x_part);
              mma_bf16(sum, a0, b.x, b.y);
              mma_bf16(sum, a1, b.z, b.w);
            }
            xa += x_step;
          }
          const float s0v = __uint_as_float(ST == kScalesBF16 ? h.scale[0][half] << 16 : h.scale[0][half]);
          const float s1v = __uint_as_float(ST == kScalesBF16 ? h.scale[1][half] << 16 : h.scale[1][half]);
          acc[0] += s0v * sum[0], acc[1] += s0v * sum[1];
          acc[2] += s1v * sum[2], acc[3] += s1v * sum[3];
        }
      }
      if (s0 + q + kAhead < W.steps) request(h);
      s += W.team;
      if (s >= W.rounds * W.team) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 1);
          acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 2);
        }
        if (tig == 0) {
          float* q_at = red + warp * 128 + gid;
          q_at[0] = acc[0], q_at[16] = acc[1], q_at[8] = acc[2], q_at[24] = acc[3];
        }
        acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
        team_sync(my_team, W.team * 32);
        head_store<1>(A, red + my_team * W.team * 128, W.in_team * 32 + lane, W.team * 32, n0, cols, tile);
        team_sync(my_team, W.team * 32);
        s = W.in_team;
        tile += W.stride;
      }
    }
  }
}

}  // namespace gls
