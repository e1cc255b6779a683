// gls_host.cuh -- what the host side of the operators next to the sampler shares.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace gls {

// SMs of the current device, looked up once per device; 148 (B200) when none can be queried
static int sm_count() {
  constexpr int kMaxDev = 64;
  static std::atomic<int> cache[kMaxDev];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDev) {
    (void)cudaGetLastError();
    return 148;
  }
  n = cache[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
    (void)cudaGetLastError();
    return 148;
  }
  cache[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Whether two sets of rows share memory: n rows of `len` bytes from p, `pitch` bytes apart, and m of `mlen` from
// q.  Rows of one pitch may lie side by side (columns of one buffer); where the pitches differ, sets whose
// stretches of memory meet are taken to share some.
static bool rows_meet(const void* p, int64_t n, int64_t pitch, int64_t len, const void* q, int64_t m, int64_t mpitch,
                      int64_t mlen) {
  typedef __int128 wide;  // a stride may be anything
  if (n == 1) pitch = mpitch;
  if (m == 1) mpitch = pitch;
  const wide a = (wide)(uintptr_t)p, b = (wide)(uintptr_t)q;
  if (a + (n - 1) * (wide)pitch + len <= b || b + (m - 1) * (wide)mpitch + mlen <= a) return false;
  if (pitch != mpitch || (n == 1 && m == 1)) return true;
  const wide r = ((b - a) % pitch + pitch) % pitch;  // a row of q begins r behind one of p
  return r < len || r + mlen > pitch;
}

}  // namespace gls
