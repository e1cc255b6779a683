// gls_head_wide.cuh -- logits of more hidden states than gls_int4.cuh's kernel takes at once: the same product on the
// 5th-generation tensor cores (tcgen05), up to 64 hidden states per pass over the table.
//
// 128 table rows are the accumulator's 128 lanes, a lane's thread has one row: it reads the row's codes from shared
// memory, turns them into bf16 differences to their zero (exact), and writes them to tensor memory as the first operand.  The
// second operand are the hidden states, in shared memory in the order of columns that masks and shifts leave.
// The products of one group of columns end up in an accumulator of their own, which the same thread reads back, multiplies
// by the group's scale and adds to its 64 sums in fp32: the scale never meets a rounding to fewer bits.  The tensor pipe
// takes 8 instructions of 128 x 64 x 16 per 128 columns; the conversion, 11 operations per 8 codes, and the 64 multiply-adds
// per group bind the kernel.
//
// A CTA has two warpgroups of that kind, each with 128 rows, which share the hidden states' tiles, and a third one: a
// thread that requests the codes, one that requests the hidden states (both by tensor copies), one that issues the
// products.  Everything is double buffered: while a group's product runs, its warpgroup converts the next group.  The hidden
// states are put in order (and fp32 ones split into three bf16 parts) by a small kernel before: two warps of
// each CTA that did so on the way took 1130 us where the copies take a fraction of it.
#pragma once
#include "gls_int4.cuh"

namespace gls {

constexpr int kWideThreads = 384, kWideCodeStages = 4, kWideRows = 128;

struct WideShared {
  // offsets in bytes; tiles on 1024-byte boundaries
  static constexpr int kCodes = 0;                                                     // [warpgroup][stage][128 rows][64]
  static constexpr int kX = 2 * kWideCodeStages * 8192;
  static __host__ __device__ constexpr int x_stage(int nb, int parts) { return parts * 2 * nb * 16 * 128; }  // [part][panel][row][128]
  static __host__ __device__ constexpr int x_stages(int parts) { return parts == 1 ? 4 : 2; }
  static __host__ __device__ constexpr int barriers(int nb, int parts) { return kX + x_stages(parts) * x_stage(nb, parts); }
  static __host__ __device__ constexpr int total(int nb, int parts) { return 1024 + barriers(nb, parts) + 264; }  // the first kilobyte: up to a boundary
};

__device__ __forceinline__ void barrier_arrive(uint32_t at) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(at) : "memory");
}
__device__ __forceinline__ void tensor_commit(uint32_t at) {  // arrives when the products issued so far are done
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(at) : "memory");
}
__device__ __forceinline__ void tensor_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_store16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tensor_load16(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
}
// D (tensor memory) (+)= A (tensor memory) x B (shared memory): bf16, fp32 sums
__device__ __forceinline__ void tensor_product(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a),
      "l"(b), "r"(kind), "r"((uint32_t)add)
      : "memory");
}
// Rows of 128 bytes, 16-byte words exchanged by the row's lowest three bits, eight rows after eight rows
__device__ __forceinline__ uint64_t tensor_tile(uint32_t at) {
  return (uint64_t)(at >> 4 & 0x3fffu) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// Hidden states -> [pass][part][kN][chunks * 128] bf16, zeros beyond N and D, within 8 columns in the order 0 4 1 5 2 6 3 7.
template <int PARTS>
__global__ void __launch_bounds__(256) head_order_kernel(const HeadArgs A, int kn, int passes, uint4* to) {
  asm volatile("griddepcontrol.launch_dependents;");
  const int words = A.chunks * 16;
  const long long all = (long long)passes * kn * words;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const int word = (int)(i % words);
    const long long n = i / words, d = (long long)word * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.f;
      if (n < A.N && d + e < A.T.D) {
        const long long at = n * A.x_stride + d + e;
        v[e] = PARTS == 1 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)A.x + at) << 16) : __ldg((const float*)A.x + at);
      }
    }
    const long long pass = n / kn, row = n % kn;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = PARTS == 1 ? __float_as_uint(v[e]) >> 16 : take_bf16(v[e]);
      to[((pass * PARTS + part) * kn + row) * words + word] =
          make_uint4(h[0] | h[4] << 16, h[1] | h[5] << 16, h[2] | h[6] << 16, h[3] | h[7] << 16);
    }
  }
}

// NB: 16 hidden states each; GPC: groups per 128 columns
template <int NB, int GPC, int PARTS>
__global__ void __launch_bounds__(kWideThreads, 1) head_wide_kernel(const HeadArgs A, const __grid_constant__ CUtensorMap codes,
                                                                   const __grid_constant__ CUtensorMap hidden) {
  extern __shared__ __align__(1024) char wide_shared[];
  constexpr int kN = 16 * NB, kXStages = WideShared::x_stages(PARTS), kXStage = WideShared::x_stage(NB, PARTS);
  constexpr int kSteps = 8 / GPC;   // products of 16 columns per group
  constexpr int kWords = 16 / GPC;  // words of 8 codes per group and row
  const Int4Table& T = A.T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wg = warp >> 2;  // warpgroup 2 serves the other two
  const uint32_t base = ((uint32_t)__cvta_generic_to_shared(wide_shared) + 1023u) & ~1023u;
  const uint32_t bars = base + WideShared::barriers(NB, PARTS);
  auto code_full = [&](int w, int s) { return bars + (w * kWideCodeStages + s) * 8; };
  auto code_free = [&](int w, int s) { return bars + 64 + (w * kWideCodeStages + s) * 8; };
  auto x_full = [&](int s) { return bars + 128 + s * 8; };
  auto x_free = [&](int s) { return bars + 160 + s * 8; };
  auto a_full = [&](int w, int s) { return bars + 192 + (w * 2 + s) * 8; };
  auto d_full = [&](int w, int s) { return bars + 224 + (w * 2 + s) * 8; };
  const uint32_t tensor_at = bars + 256;  // where the tensor memory's address is put
  volatile int& lost = *(volatile int*)(wide_shared + (bars + 260 - (uint32_t)__cvta_generic_to_shared(wide_shared)));
  // lost: a wait ran out; nothing waits any more and the results are NaN

  if (threadIdx.x == 0) {
    lost = 0;
    for (int w = 0; w < 2; ++w) {
      for (int s = 0; s < kWideCodeStages; ++s) barrier_init(code_full(w, s), 1), barrier_init(code_free(w, s), 4);
      for (int s = 0; s < 2; ++s) barrier_init(a_full(w, s), 4), barrier_init(d_full(w, s), 1);
    }
    for (int s = 0; s < kXStages; ++s) barrier_init(x_full(s), 1), barrier_init(x_free(s), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tensor_at) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tensor_before();
  __syncthreads();
  tensor_after();
  uint32_t tm;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tm) : "r"(tensor_at));
  auto wait = [&](uint32_t at, uint32_t parity) {
    if (lost) return;
    if (!barrier_wait(at, parity)) lost = 1;
  };

  const int n0 = blockIdx.y * kN, cols = min(kN, A.N - n0);
  const long long pairs = (T.V + 2 * kWideRows - 1) / (2 * kWideRows);  // tiles of 256 rows
  const int mine = (int)((pairs - blockIdx.x + gridDim.x - 1) / gridDim.x);
  const int groups = T.G;  // per row; the last chunk may have fewer than GPC

  if (wg < 2) {
    // ---- a row per thread: codes -> first operand; accumulators -> sums
    const int w4 = warp & 3;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    const uint32_t a_at = tm + lanes + wg * 128, d_at = tm + lanes + 256 + wg * 128;  // two buffers of 64 columns each
    const int row = w4 * 32 + lane;
    long long unit = 0;   // groups so far
    long long chunk = 0;  // chunks so far
    for (int i = 0; i < mine; ++i) {
      const long long tile = blockIdx.x + (long long)i * gridDim.x, v = (tile * 2 + wg) * kWideRows + row;
      const long long vr = v < T.V ? v : T.V - 1;
      const char* const sp = (const char*)T.scales + vr * T.scale_stride * (T.scale_bf16 ? 2 : 4);
      const uint8_t* const zp = T.zeros ? T.zeros + vr * T.zero_stride : nullptr;
      auto scale_of = [&](int g) {
        return T.scale_bf16 ? __uint_as_float((uint32_t)__ldg((const unsigned short*)sp + g) << 16) : __ldg((const float*)sp + g);
      };
      auto zero_of = [&](int g) { return zp ? (uint32_t)__ldg(zp + g) & 15u : 8u; };
      float acc[kN];
#pragma unroll
      for (int n = 0; n < kN; ++n) acc[n] = 0.f;
      float scale = 0.f, next_scale = scale_of(0);
      uint32_t next_zero = zero_of(0);
      auto add_up = [&](long long u, float s) {  // the sums of group u, times its scale
        wait(d_full(wg, (int)(u & 1)), (uint32_t)(u >> 1) & 1u);
        __syncwarp();
        tensor_after();
        constexpr int kAt = NB % 2 ? 1 : 2;  // sets of 16 read at a time
#pragma unroll
        for (int h = 0; h < NB; h += kAt) {
          uint32_t d[16 * kAt];
#pragma unroll
          for (int j = 0; j < kAt; ++j) tensor_load16(d_at + (uint32_t)(u & 1) * 64 + (h + j) * 16, d + 16 * j);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int n = 0; n < 16 * kAt; ++n) acc[h * 16 + n] = fmaf(s, __uint_as_float(d[n]), acc[h * 16 + n]);
        }
        tensor_before();
      };
      for (int g = 0; g < groups; ++g, ++unit) {
        const int sub = g & (GPC - 1), stage = (int)(chunk % kWideCodeStages);
        const float last_scale = scale;
        scale = next_scale;
        const uint32_t z = (0x4300u | next_zero) * 0x10001u;
        if (g + 1 < groups) next_scale = scale_of(g + 1), next_zero = zero_of(g + 1);
        if (sub == 0) wait(code_full(wg, stage), (uint32_t)(chunk / kWideCodeStages) & 1u);
        __syncwarp();
        const uint32_t at = base + WideShared::kCodes + (wg * kWideCodeStages + stage) * 8192 + row * 64;
#pragma unroll
        for (int q = 0; q < kWords / 4; ++q) {
          const int word = sub * (kWords / 4) + q;  // of 16 bytes
          const uint4 c = lds16(at + ((word ^ (row >> 1 & 3)) << 4));
          const uint32_t w[4] = {c.x, c.y, c.z, c.w};
          uint32_t p[16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t t[4];
            int4_pairs(w[j], z, t);
#pragma unroll
            for (int k = 0; k < 4; ++k) p[4 * j + k] = t[k];
          }
          tensor_store16(a_at + (uint32_t)(unit & 1) * 64 + q * 16, p);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tensor_before();
        __syncwarp();
        if (lane == 0) {
          barrier_arrive(a_full(wg, (int)(unit & 1)));
          if (sub == GPC - 1 || g == groups - 1) barrier_arrive(code_free(wg, stage));
        }
        if (sub == GPC - 1 || g == groups - 1) ++chunk;
        if (g > 0) add_up(unit - 1, last_scale);
      }
      add_up(unit - 1, scale);
      const float bad = lost ? __uint_as_float(0x7fc00000u) : 0.f;
      if (v < T.V) {
#pragma unroll
        for (int n = 0; n < kN; ++n)
          if (n < cols) {
            const long long o = (long long)(n0 + n) * A.out_stride + v;
            if (A.out_bf16) ((unsigned short*)A.out)[o] = (unsigned short)bf16_bits(acc[n] + bad);
            else ((float*)A.out)[o] = acc[n] + bad;
          }
      }
    }
  } else if (warp == 8) {
    // ---- codes of both warpgroups
    if (lane == 0) {
      long long chunk = 0;
      for (int i = 0; i < mine; ++i) {
        const long long tile = blockIdx.x + (long long)i * gridDim.x;
        for (int c = 0; c < A.chunks; ++c, ++chunk) {
          const int s = (int)(chunk % kWideCodeStages);
          for (int w = 0; w < 2; ++w) {
            if (chunk >= kWideCodeStages) wait(code_free(w, s), (uint32_t)(chunk / kWideCodeStages - 1) & 1u);
            if (lost) continue;
            barrier_expect(code_full(w, s), 8192);
            copy_box(base + WideShared::kCodes + (w * kWideCodeStages + s) * 8192, &codes, c * 64, (int)((tile * 2 + w) * kWideRows), code_full(w, s));
          }
        }
      }
      // nothing of its own is under way when the CTA ends: the warpgroups have waited for every copy, unless a wait ran out
      if (lost)
        for (int w = 0; w < 2; ++w)
          for (int s = 0; s < kWideCodeStages; ++s)
            for (uint32_t parity = 0; parity < 2; ++parity) (void)barrier_wait(code_full(w, s), parity);
    }
  } else if (warp == 9) {
    // ---- the products
    if (lane == 0) {
      constexpr uint32_t kind = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kWideRows >> 4) << 24;
      long long unit = 0, chunk = 0;
      for (int i = 0; i < mine; ++i) {
        for (int c = 0; c < A.chunks; ++c, ++chunk) {
          const int xs = (int)(chunk % kXStages);
          wait(x_full(xs), (uint32_t)(chunk / kXStages) & 1u);
          for (int sub = 0; sub < GPC && c * GPC + sub < groups; ++sub, ++unit) {
            const int b = (int)(unit & 1);
            for (int w = 0; w < 2; ++w) {
              wait(a_full(w, b), (uint32_t)(unit >> 1) & 1u);
              tensor_after();
              if (!lost) {
#pragma unroll
                for (int part = 0; part < PARTS; ++part)
#pragma unroll
                  for (int k = 0; k < kSteps; ++k) {
                    const int kk = sub * kSteps + k;  // of eight; four to a panel
                    const uint32_t x = base + WideShared::kX + xs * kXStage + (part * 2 + (kk >> 2)) * (kN * 128) + (kk & 3) * 32;
                    tensor_product(tm + 256 + w * 128 + b * 64, tm + w * 128 + b * 64 + k * 8, tensor_tile(x), kind, part + k > 0);
                  }
              }
              tensor_commit(d_full(w, b));
            }
          }
          tensor_commit(x_free(xs));
        }
      }
    }
  } else if (warp == 10) {
    // ---- the hidden states
    if (lane == 0) {
      asm volatile("griddepcontrol.wait;" ::: "memory");  // the kernel that puts them in order
      long long chunk = 0;
      for (int i = 0; i < mine; ++i) {
        for (int c = 0; c < A.chunks; ++c, ++chunk) {
          const int xs = (int)(chunk % kXStages);
          if (chunk >= kXStages) wait(x_free(xs), (uint32_t)(chunk / kXStages - 1) & 1u);
          if (lost) continue;
          barrier_expect(x_full(xs), (uint32_t)kXStage);
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int panel = 0; panel < 2; ++panel)
              copy_box(base + WideShared::kX + xs * kXStage + (part * 2 + panel) * (kN * 128), &hidden, c * 128 + panel * 64,
                         ((int)blockIdx.y * PARTS + part) * kN, x_full(xs));
        }
      }
      if (lost)
        for (int xs = 0; xs < kXStages; ++xs)
          for (uint32_t parity = 0; parity < 2; ++parity) (void)barrier_wait(x_full(xs), parity);
    }
  }
  __syncwarp();
  tensor_before();
  __syncthreads();
  tensor_after();
  __syncwarp();
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
}

}  // namespace gls
