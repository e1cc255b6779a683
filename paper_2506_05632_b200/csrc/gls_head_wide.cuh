// gls_head_wide.cuh -- logits of more hidden states than gls_int4.cuh's kernel takes at once: the same product on the
// 5th-generation tensor cores (tcgen05), up to 64 hidden states per pass over the table.
//
// 128 table rows are the accumulator's 128 lanes, a lane's thread has one row: it reads the row's codes from shared
// memory, turns them into bf16 differences to their zero (exact), and writes them to tensor memory as the first operand.  The
// second operand are the hidden states, in shared memory in the order of columns that masks and shifts leave.
// The products of one group of columns end up in an accumulator of their own, which the same thread reads back, multiplies
// by the group's scale and adds to its 64 sums in fp32: the scale never meets a rounding to fewer bits.  The tensor pipe
// takes 8 instructions of 128 x 64 x 16 per 128 columns; the conversion, 11 operations per 8 codes, and the 64 multiply-adds
// per row and group, and what they wait for, bind the kernel.
//
// A CTA has two tiles of 128 rows at a time, which share the hidden states' tiles, and two warpgroups for each.  A
// warpgroup takes every other group of columns of its tile: while one waits for its group's products the other converts
// the next group (one warpgroup a tile, or two that share each group, wait most of the time: 251 us for 64 hidden states,
// 152064 x 4096).  At the tile's end the two exchange halves of their sums.  Three more warps serve them: one that requests codes
// and hidden states (tensor copies), one for either tile that issues the products.  The hidden states are put in order (and
// fp32 ones split into three bf16 parts) by a small kernel before.
#pragma once
#include "gls_int4.cuh"

namespace gls {

constexpr int kWideThreads = 640, kWideCodeStages = 4, kWideRows = 128;

struct WideShared {
  // offsets in bytes; tiles on 1024-byte boundaries
  static constexpr int kCodes = 0;                                                     // [tile][stage][128 rows][64]
  static constexpr int kX = 2 * kWideCodeStages * 8192;
  static __host__ __device__ constexpr int x_stage(int nb, int parts) { return parts * 2 * nb * 16 * 128; }  // [part][panel][row][128]
  static __host__ __device__ constexpr int x_stages(int parts) { return parts == 1 ? 4 : 2; }
  static __host__ __device__ constexpr int barriers(int nb, int parts) { return kX + x_stages(parts) * x_stage(nb, parts); }
  // scales and zeros of eight groups [8][512 threads] 8 bytes; at a tile's end, among the places of
  // the tile's own threads, sums on their way [16][128] from either side
  static __host__ __device__ constexpr int scales(int nb, int parts) { return barriers(nb, parts) + 512; }
  static __host__ __device__ constexpr int total(int nb, int parts) { return 1024 + scales(nb, parts) + 32768; }  // the first kilobyte: up to a boundary
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
  constexpr int kHalf = kN / 2;
  constexpr int kSteps = 8 / GPC;   // products of 16 columns per group
  constexpr int kWords = 16 / GPC;  // words of 8 codes per group and row
  const Int4Table& T = A.T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pair = warp >> 3, side = warp >> 2 & 1;  // a tile's warpgroups
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
      for (int s = 0; s < kWideCodeStages; ++s) barrier_init(code_full(w, s), 1), barrier_init(code_free(w, s), GPC == 1 ? 4 : 8);
      for (int s = 0; s < 2; ++s) barrier_init(a_full(w, s), 4), barrier_init(d_full(w, s), 1);
    }
    for (int s = 0; s < kXStages; ++s) barrier_init(x_full(s), 1), barrier_init(x_free(s), 2);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 17) {
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

  if (pair < 2) {
    // ---- a row per thread, every other group: codes -> first operand; accumulators -> sums
    const int w4 = warp & 3, row = w4 * 32 + lane;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    const uint32_t a_at = tm + lanes + pair * 128 + side * 64, d_at = tm + lanes + 256 + pair * 128 + side * 64;
    const uint32_t slot = base + WideShared::scales(NB, PARTS) + threadIdx.x * 8;  // scales: each thread its own copy
    long long chunk = 0;  // so far, of all tiles
    uint32_t used = 0u;   // how often the buffers were
    for (int i = 0; i < mine; ++i) {
      const long long tile = blockIdx.x + (long long)i * gridDim.x, v = (tile * 2 + pair) * kWideRows + row;
      const long long vr = v < T.V ? v : T.V - 1;
      const char* const sp = (const char*)T.scales + vr * T.scale_stride * (T.scale_bf16 ? 2 : 4);
      const uint8_t* const zp = T.zeros ? T.zeros + vr * T.zero_stride : nullptr;
      // Scales and zeros of eight groups at a time: a warp's read of 32 rows is 32 lines, whatever it takes of them.
      uint32_t raw[8], zraw[2];
      auto load_block = [&](int g0) {
        zraw[0] = zraw[1] = 0x08080808u;
        if (A.vec && g0 + 8 <= groups) {
          if (T.scale_bf16) load_words<16>(raw, sp + g0 * 2);
          else load_words<32>(raw, sp + g0 * 4);
          if (zp) load_words<8>(zraw, (const char*)zp + g0);
        } else {
          if (zp) zraw[0] = zraw[1] = 0u;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool in = g0 + j < groups;
            if (T.scale_bf16) {
              const uint32_t h = in ? (uint32_t)__ldg((const unsigned short*)sp + g0 + j) : 0u;
              if (j & 1) raw[j >> 1] |= h << 16;
              else raw[j >> 1] = h;
            } else {
              raw[j] = in ? __ldg((const uint32_t*)sp + g0 + j) : 0u;
            }
            if (zp && in) zraw[j >> 2] |= (uint32_t)__ldg(zp + g0 + j) << (8 * (j & 3));
          }
        }
      };
      auto store_block = [&]() {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t f = !T.scale_bf16 ? raw[j] : j & 1 ? raw[j >> 1] & 0xffff0000u : raw[j >> 1] << 16;
          const uint32_t z = __byte_perm(zraw[j >> 2] & 0x0f0f0f0fu, 0x43u, 0x4040u | (uint32_t)(j & 3) * 0x0101u);
          asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(slot + j * 4096), "r"(f), "r"(z) : "memory");
        }
      };
      load_block(0);
      float acc[kN];
#pragma unroll
      for (int n = 0; n < kN; ++n) acc[n] = 0.f;
      for (int c = 0; c < A.chunks; ++c, ++chunk) {
        if (GPC == 1 && (c & 1) != side) continue;
        const int stage = (int)(chunk % kWideCodeStages);
        wait(code_full(pair, stage), (uint32_t)(chunk / kWideCodeStages) & 1u);
        __syncwarp();
        const uint32_t at = base + WideShared::kCodes + (pair * kWideCodeStages + stage) * 8192 + row * 64;
#pragma unroll
        for (int sub = GPC == 1 ? 0 : side; sub < GPC; sub += 2) {
          const int g = c * GPC + sub;
          if (g < groups) {
            if ((g & 7) == side) store_block();
            const uint2 sz = lds8(slot + (g & 7) * 4096);
            if ((g & 7) == side + 2 && g - side + 6 < groups) load_block(g - side + 6);
#pragma unroll
            for (int q = 0; q < kWords / 4; ++q) {
              const int word = sub * (kWords / 4) + q;  // of 16 bytes
              const uint4 k4 = lds16(at + ((word ^ (row >> 1 & 3)) << 4));
              const uint32_t w[4] = {k4.x, k4.y, k4.z, k4.w};
              uint32_t p[16];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t t[4];
                int4_pairs(w[j], sz.y, t);
#pragma unroll
                for (int k = 0; k < 4; ++k) p[4 * j + k] = t[k];
              }
              tensor_store16(a_at + q * 16, p);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            tensor_before();
            __syncwarp();
            if (lane == 0) {
              barrier_arrive(a_full(pair, side));
              if (GPC == 1 || sub + 2 >= GPC) barrier_arrive(code_free(pair, stage));
            }
            // the group's sums, times its scale
            const float s = __uint_as_float(sz.x);
            wait(d_full(pair, side), used & 1u);
            ++used;
            __syncwarp();
            tensor_after();
#pragma unroll
            for (int h = 0; h < NB; ++h) {
              uint32_t d[16];
              tensor_load16(d_at + h * 16, d);
              asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
              for (int n = 0; n < 16; ++n) acc[h * 16 + n] = fmaf(s, __uint_as_float(d[n]), acc[h * 16 + n]);
            }
            tensor_before();
          } else if (lane == 0 && (GPC == 1 || sub + 2 >= GPC)) {
            barrier_arrive(code_free(pair, stage));
          }
        }
      }
      // The tile's other warpgroup has the other groups' sums: each sends the half that it does not store, through the
      // scales' place, up to 16 hidden states at a time.
      const uint32_t out_box = base + WideShared::scales(NB, PARTS) + side * 16384 + pair * 2048 + row * 4;
      const uint32_t in_box = side ? out_box - 16384 : out_box + 16384;
      constexpr int kAt = kHalf < 16 ? kHalf : 16;
      auto pair_sync = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(1 + pair) : "memory"); };
      pair_sync();
#pragma unroll
      for (int from = 0; from < kHalf; from += kAt) {
#pragma unroll
        for (int n = 0; n < kAt; ++n)
          if (from + n < kHalf)
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(out_box + (n >> 2) * 4096 + (n & 3) * 512), "f"(side ? acc[from + n] : acc[kHalf + from + n]) : "memory");
        pair_sync();
#pragma unroll
        for (int n = 0; n < kAt; ++n)
          if (from + n < kHalf) {
            float y;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(y) : "r"(in_box + (n >> 2) * 4096 + (n & 3) * 512) : "memory");
            // the first warpgroup's sum is the first term on both sides
            if (side) acc[kHalf + from + n] = y + acc[kHalf + from + n];
            else acc[from + n] += y;
          }
        pair_sync();
      }
      const float bad = lost ? __uint_as_float(0x7fc00000u) : 0.f;
      if (v < T.V) {
#pragma unroll
        for (int n = 0; n < kHalf; ++n) {
          const int col = side * kHalf + n;
          const float y = (side ? acc[kHalf + n] : acc[n]) + bad;
          if (col < cols) {
            const long long o = (long long)(n0 + col) * A.out_stride + v;
            if (A.out_bf16) ((unsigned short*)A.out)[o] = (unsigned short)bf16_bits(y);
            else ((float*)A.out)[o] = y;
          }
        }
      }
    }
  } else if (warp == 16) {
    // ---- hidden states, and codes of both tiles
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the kernel that puts the hidden states in order
    uint32_t chunk = 0;
    for (int i = 0; i < mine; ++i) {
      const long long tile = blockIdx.x + (long long)i * gridDim.x;
      for (int c = 0; c < A.chunks; ++c, ++chunk) {
        const int s = (int)(chunk % kWideCodeStages), xs = (int)(chunk % kXStages);
        if (chunk >= kXStages) wait(x_free(xs), (chunk / kXStages - 1) & 1u);
        __syncwarp();
        if (!lost && elected()) {
          barrier_expect(x_full(xs), (uint32_t)kXStage);
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int panel = 0; panel < 2; ++panel)
              copy_box(base + WideShared::kX + xs * kXStage + (part * 2 + panel) * (kN * 128), &hidden, c * 128 + panel * 64,
                       ((int)blockIdx.y * PARTS + part) * kN, x_full(xs));
        }
        for (int w = 0; w < 2; ++w) {
          if (chunk >= kWideCodeStages) wait(code_free(w, s), (chunk / kWideCodeStages - 1) & 1u);
          __syncwarp();
          if (!lost && elected()) {
            barrier_expect(code_full(w, s), 8192);
            copy_box(base + WideShared::kCodes + (w * kWideCodeStages + s) * 8192, &codes, c * 64, (int)((tile * 2 + w) * kWideRows), code_full(w, s));
          }
        }
      }
    }
    // nothing of its own is under way when the CTA ends: the others have waited for every copy, unless a wait ran out
    if (lost) {
      for (uint32_t parity = 0; parity < 2; ++parity) {
        for (int s = 0; s < kWideCodeStages; ++s) (void)barrier_wait(code_full(0, s), parity), (void)barrier_wait(code_full(1, s), parity);
        for (int xs = 0; xs < kXStages; ++xs) (void)barrier_wait(x_full(xs), parity);
      }
    }
  } else if (warp < 19) {
    // ---- the products of a tile
    const int w = warp - 17;
    constexpr uint32_t kind = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kWideRows >> 4) << 24;
    uint32_t chunk = 0, used[2] = {0u, 0u};  // how often the buffers of either side were
    for (int i = 0; i < mine; ++i) {
      for (int c = 0; c < A.chunks; ++c, ++chunk) {
        const int xs = (int)(chunk % kXStages);
        wait(x_full(xs), (chunk / kXStages) & 1u);
        const uint64_t x_tile = tensor_tile(base + WideShared::kX + xs * kXStage);
#pragma unroll
        for (int sub = 0; sub < GPC; ++sub) {
          if (c * GPC + sub >= groups) break;
          const int b = GPC == 1 ? c & 1 : sub & 1;
          const uint32_t phase = (b ? used[1] : used[0]) & 1u;
          if (b) ++used[1];
          else ++used[0];
          wait(a_full(w, b), phase);
          __syncwarp();
          tensor_after();
          if (elected()) {
            if (!lost) {
#pragma unroll
              for (int part = 0; part < PARTS; ++part)
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                  const int kk = sub * kSteps + k;  // of eight; four to a panel
                  tensor_product(tm + 256 + w * 128 + b * 64, tm + w * 128 + b * 64 + k * 8,
                                 x_tile + (uint64_t)(((part * 2 + (kk >> 2)) * (kN * 128) + (kk & 3) * 32) >> 4), kind, part + k > 0);
                }
            }
            tensor_commit(d_full(w, b));
          }
        }
        if (elected()) tensor_commit(x_free(xs));
      }
    }
  }
  __syncwarp();
  tensor_before();
  __syncthreads();
  tensor_after();
  __syncwarp();
  if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
}

}  // namespace gls
