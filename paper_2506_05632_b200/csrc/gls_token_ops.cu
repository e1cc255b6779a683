// gls_token_ops.cu -- C ABI of the operators next to the sampler (see include/gls.h): log
// probabilities of tokens with entropy and alternatives and their gradient, the embedding lookup
// and its gradient.
#include <atomic>
#include <cmath>
#include <cstring>

#include "../../include/gls.h"
#include "gls_embed.cuh"

namespace gls {

static_assert(kDevBadToken == GLS_DEV_BAD_TOKEN && kScoreMaxG == GLS_MAX_GIVEN && kMaxK == GLS_MAX_K, "header");

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

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

static bool score_sizes_ok(int B, int K, int J, int64_t V) {
  return B > 0 && K > 0 && K <= GLS_MAX_K && J > 0 && V > 0 && V < (1LL << 31) - 65536 &&
         (long long)B * K * J < (1LL << 31) / 64;
}
static int rows_ok(const gls_rows_t* r) {
  if (!r || !r->data) return GLS_ERR_INVALID_ARG;
  if (r->dtype != GLS_F32 && r->dtype != GLS_BF16) return GLS_ERR_UNSUPPORTED;
  if (((uintptr_t)r->data) % (r->dtype == GLS_F32 ? 4 : 2)) return GLS_ERR_MISALIGNED;
  return GLS_OK;
}
// Temperatures are held to a range in which a difference of logits scaled by one neither vanishes
// nor overflows before its exponential does.
static int temps_ok(float inv_temp, const float* per_draft, int K, float* out) {
  for (int k = 0; k < K; ++k) {
    const float it = per_draft ? per_draft[k] : inv_temp;
    if (!std::isfinite(it) || it <= 0.f) return GLS_ERR_INVALID_ARG;
    if (it < 1e-20f || it > 1e20f) return GLS_ERR_UNSUPPORTED;
    out[k] = it;
  }
  return GLS_OK;
}

// Which kernel scores `rows` rows of V tokens: 0, a warp per row; c > 0, a cluster of c CTAs per row.
// The times (us) are a fit to both kernels over 1 .. 8192 rows of 1000 .. 152064 tokens; a step is 4 KB of a
// row, read by one warp.  Measured, by a warp / by 1, 2, 4, 8 CTAs per row: 1 row of 152064 bf16 tokens
// 54 / 19, 14, 12, 11; 224 of 128256 53 / 23, 21, 28, 39; 1200 of 152064 96 / 86, 97, 131, 213; 2400 of 152064
// 168 / 146, 177, ..; 8192 of 152064 423 / 455, ..; 1000 of 8000 14 / 20, 40, ..
static int score_ctas(long long rows, long long V, int M, int dtype) {
  const int step = dtype == GLS_BF16 ? ScoreCfg<kBF16>::kStep : ScoreCfg<kF32>::kStep;
  const double steps = (double)((V + 15 + step - 1) / step);  // a row may start 15 elements past a boundary
  const double warps = (double)sm_count() * kScoreCtasPerSM, slots = (double)sm_count() * kClCtasPerSM;
  const double load = (double)rows / warps;
  if (M > kFineTop * steps) return 0;  // the rows kernel has a bound for these
  double least = 8.0 + steps * (load <= 1.0 ? 0.62 + load : 0.8 + 1.4 * load);
  int best = 0;
  for (int c = 1; c <= kClMaxCtas; c *= 2) {
    // a CTA's bound on the M-th logit comes from 32 maxima per step: with fewer than 2 M of them so many
    // tokens reach it that the buffers overflow and the radix selection has to read the row again
    if (c > 1 && 16.0 * steps < (double)c * M) break;
    const double waves = (double)rows * c / slots, each = std::ceil(steps / (c * kClWarps));
    const double t = 9.0 + (waves <= 1.0 ? each * (0.5 + 1.2 * waves) : (waves + 0.35) * (4.0 + 1.5 * each));
    if (t < least) {
      least = t;
      best = c;
    }
  }
  return best;
}

template <int DT, bool ENT>
static cudaError_t launch_score(const ScoreArgs& A, int ctas, cudaStream_t st) {
  if (ctas == 0) {
    const long long cap = (long long)sm_count() * kScoreCtasPerSM;
    const size_t smem = A.M > 0 ? sizeof(RowShared) : 0;
    score_rows_kernel<DT, ENT><<<(unsigned)(A.rows < cap ? A.rows : cap), 32, smem, st>>>(A);
    return cudaGetLastError();
  }
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(A.rows * ctas));
  cfg.blockDim = dim3(kClThreads);
  cfg.dynamicSmemBytes = sizeof(ClusterShared);
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, score_cluster_kernel<DT, ENT>, A, ctas);
}

static int run_score(ScoreArgs& A, const gls_rows_t* rows, int ctas, cudaStream_t st) {
  A.data = rows->data;
  A.sb = rows->stride_b;
  A.sk = rows->stride_k;
  A.sj = rows->stride_j;
  const bool bf = rows->dtype == GLS_BF16, ent = A.out_ent != nullptr;
  const cudaError_t err = bf ? (ent ? launch_score<kBF16, true>(A, ctas, st) : launch_score<kBF16, false>(A, ctas, st))
                             : (ent ? launch_score<kF32, true>(A, ctas, st) : launch_score<kF32, false>(A, ctas, st));
  return err == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

}  // namespace gls

using namespace gls;

namespace gls {
// the range-check record of this translation unit's kernels (gls_debug_bounds adds it to its own)
int token_ops_bounds(uint32_t out[4]) {
#ifdef GLS_DEBUG_BOUNDS
  return cudaMemcpyFromSymbol(out, g_bounds_fault, 4 * sizeof(uint32_t)) == cudaSuccess ? 1 : -1;
#else
  out[0] = out[1] = out[2] = out[3] = 0u;
  return 0;
#endif
}
}  // namespace gls

extern "C" {

int gls_token_logprobs(const gls_rows_t* logits, int B, int K, int J, int64_t V, float inv_temp,
                       const float* inv_temp_per_draft_host, const int32_t* tokens, int G, int M,
                       float* out_logprobs, float* out_lse, float* out_lse_tail, float* out_entropy,
                       int32_t* out_top_ids, float* out_top_logprobs, uint32_t* device_status,
                       void* stream) {
  if (!score_sizes_ok(B, K, J, V) || G < 0 || G > GLS_MAX_GIVEN || M < 0 || M > kScoreMaxM || !out_lse)
    return GLS_ERR_INVALID_ARG;
  if ((G > 0 && (!tokens || !out_logprobs)) || (M > 0 && (!out_top_ids || !out_top_logprobs)))
    return GLS_ERR_INVALID_ARG;
  int rc = rows_ok(logits);
  if (rc != GLS_OK) return rc;
  ScoreArgs A;
  std::memset(&A, 0, sizeof(A));
  rc = temps_ok(inv_temp, inv_temp_per_draft_host, K, A.inv_t);
  if (rc != GLS_OK) return rc;
  A.K = K;
  A.J = J;
  A.V = (int)V;
  A.M = M;
  A.G = G;
  A.rows = (long long)B * K * J;
  A.tokens = tokens;
  A.out_lp = out_logprobs;
  A.out_lse = out_lse;
  A.out_tail = out_lse_tail;
  A.out_ent = out_entropy;
  A.top_ids = out_top_ids;
  A.top_lp = out_top_logprobs;
  A.status = device_status;
  return run_score(A, logits, score_ctas(A.rows, V, M, logits->dtype), (cudaStream_t)stream);
}

int gls_emitted_logprobs(const gls_rows_t* target_logits, int B, int K, int L, int64_t V, float inv_temp,
                         const int32_t* tokens, const uint8_t* accept, uint32_t flags, int M,
                         float* out_logprobs, float* out_lse, float* out_entropy, int32_t* out_top_ids,
                         float* out_top_logprobs, uint32_t* device_status, void* stream) {
  if (flags & ~(GLS_NO_BONUS | GLS_COMBINE_ALL)) return GLS_ERR_INVALID_ARG;
  if (L < 0 || L >= (1 << 30)) return GLS_ERR_INVALID_ARG;
  const int J = L + ((flags & GLS_NO_BONUS) ? 0 : 1);
  if (!score_sizes_ok(B, K, J, V) || M < 0 || M > kScoreMaxM || !tokens || !out_logprobs || !out_lse)
    return GLS_ERR_INVALID_ARG;
  if ((J > 1 && !accept) || (M > 0 && (!out_top_ids || !out_top_logprobs))) return GLS_ERR_INVALID_ARG;
  int rc = rows_ok(target_logits);
  if (rc != GLS_OK) return rc;
  ScoreArgs A;
  std::memset(&A, 0, sizeof(A));
  rc = temps_ok(inv_temp, nullptr, K, A.inv_t);
  if (rc != GLS_OK) return rc;
  A.K = K;
  A.J = J;
  A.V = (int)V;
  A.M = M;
  A.G = 1;
  A.emitted = 1;
  A.L = L;
  A.accept = accept;
  A.rows = (long long)B * J;
  A.tokens = tokens;
  A.out_lp = out_logprobs;
  A.out_lse = out_lse;
  A.out_ent = out_entropy;
  A.top_ids = out_top_ids;
  A.top_lp = out_top_logprobs;
  A.status = device_status;
  // between one row per sequence and J are read
  return run_score(A, target_logits, score_ctas((long long)B * (J + 1) / 2, V, M, target_logits->dtype),
                   (cudaStream_t)stream);
}

int gls_token_logprobs_backward(const gls_rows_t* logits, int B, int K, int J, int64_t V, float inv_temp,
                                const float* inv_temp_per_draft_host, const int32_t* tokens, int G,
                                const int32_t* top_ids, int M, const float* lse, const float* lse_tail,
                                const float* entropy, const float* grad_logprobs, const float* grad_lse,
                                const float* grad_entropy, const float* grad_top_logprobs,
                                const gls_rows_t* grad_logits, void* stream) {
  if (!score_sizes_ok(B, K, J, V) || G < 0 || G > GLS_MAX_GIVEN || M < 0 || M > kScoreMaxM || !lse)
    return GLS_ERR_INVALID_ARG;
  if ((grad_logprobs && G > 0 && !tokens) || (grad_top_logprobs && M > 0 && !top_ids) || (grad_entropy && !entropy))
    return GLS_ERR_INVALID_ARG;
  int rc = rows_ok(logits);
  if (rc == GLS_OK) rc = rows_ok(grad_logits);
  if (rc != GLS_OK) return rc;
  if (logits->dtype != grad_logits->dtype) return GLS_ERR_UNSUPPORTED;
  // every element of the gradient has a place of its own, and not that of a logit
  if (grad_logits->data == logits->data || (B > 1 && grad_logits->stride_b == 0) ||
      (K > 1 && grad_logits->stride_k == 0) || (J > 1 && grad_logits->stride_j == 0))
    return GLS_ERR_INVALID_ARG;
  ScoreGradArgs A;
  std::memset(&A, 0, sizeof(A));
  rc = temps_ok(inv_temp, inv_temp_per_draft_host, K, A.inv_t);
  if (rc != GLS_OK) return rc;
  A.data = logits->data;
  A.sb = logits->stride_b;
  A.sk = logits->stride_k;
  A.sj = logits->stride_j;
  A.grad = (void*)grad_logits->data;
  A.gb = grad_logits->stride_b;
  A.gk = grad_logits->stride_k;
  A.gj = grad_logits->stride_j;
  A.K = K;
  A.J = J;
  A.V = (int)V;
  A.M = M;
  A.G = G;
  A.rows = (long long)B * K * J;
  A.tokens = tokens;
  A.top_ids = top_ids;
  A.lse = lse;
  A.tail = lse_tail;
  A.ent = entropy;
  A.g_lp = G > 0 ? grad_logprobs : nullptr;
  A.g_lse = grad_lse;
  A.g_ent = grad_entropy;
  A.g_top = M > 0 ? grad_top_logprobs : nullptr;
  const bool bf = logits->dtype == GLS_BF16;
  for (int k = 0; k < K; ++k) A.temp[k] = 1.0f / A.inv_t[k];
  // chunks of up to 64 KB of a row, shorter where there would not be one for every resident CTA (640
  // rows of 50257 bf16 tokens: chunks of 16 KB 31 us, of 64 KB 26)
  const long long turn = (long long)kGradThreads * kGradVecs * (bf ? 16 : 8), turns = (V + 15 + turn - 1) / turn;
  const long long want = (long long)sm_count() * kGradCtasPerSM;
  long long iters = turns * A.rows / want;
  iters = iters < 1 ? 1 : iters > 4 ? 4 : iters;
  A.iters = (int)iters;
  A.chunks = (int)((turns + iters - 1) / iters);
  const long long items = A.rows * A.chunks;
  const int grid = (int)(items < (1 << 20) ? items : (1 << 20));
  cudaStream_t st = (cudaStream_t)stream;
  if (bf && grad_entropy) score_grad_kernel<kBF16, true><<<grid, kGradThreads, 0, st>>>(A);
  else if (bf) score_grad_kernel<kBF16, false><<<grid, kGradThreads, 0, st>>>(A);
  else if (grad_entropy) score_grad_kernel<kF32, true><<<grid, kGradThreads, 0, st>>>(A);
  else score_grad_kernel<kF32, false><<<grid, kGradThreads, 0, st>>>(A);
  return cudaGetLastError() == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

int gls_embed_tokens(const void* table, int dtype, int64_t table_stride, int64_t V, int64_t D,
                     const int32_t* tokens, int64_t N, float scale, void* out, int64_t out_stride,
                     uint32_t* device_status, void* stream) {
  if (V <= 0 || V >= (1LL << 31) || D <= 0 || D >= (1LL << 31) || N < 0 || N >= (1LL << 31) || !std::isfinite(scale))
    return GLS_ERR_INVALID_ARG;
  if (dtype != GLS_F32 && dtype != GLS_BF16) return GLS_ERR_UNSUPPORTED;
  if (N == 0) return GLS_OK;
  if (!table || !tokens || !out || (V > 1 && table_stride < D) || (N > 1 && out_stride < D)) return GLS_ERR_INVALID_ARG;
  const int es = dtype == GLS_F32 ? 4 : 2;
  if ((uintptr_t)table % es || (uintptr_t)out % es) return GLS_ERR_MISALIGNED;
  // the table is read while the rows are written
  if (rows_meet(table, V, table_stride * es, D * es, out, N, out_stride * es, D * es)) return GLS_ERR_INVALID_ARG;
  EmbedArgs A;
  A.table = (const char*)table;
  A.table_stride = table_stride;
  A.out = (char*)out;
  A.out_stride = out_stride;
  A.tokens = tokens;
  A.N = N;
  A.V = V;
  A.D = D;
  A.scale = scale;
  A.status = device_status;
  cudaStream_t st = (cudaStream_t)stream;
  const bool vec = D * es % 16 == 0 && table_stride * es % 16 == 0 && out_stride * es % 16 == 0 &&
                   (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0;
  const uint32_t per_row = (uint32_t)(vec ? D * es / 16 : row_pieces(D * es, es));
  const bool rows_long = per_row >= kEmbedLongRow;
  const long long per_cta = rows_long ? kEmbedThreads / 32 : kEmbedThreads * kEmbedUnits;
  const long long units = rows_long ? N * ((per_row + 32 * kEmbedUnits - 1) / (32 * kEmbedUnits)) : N * per_row;
  const long long want = (units + per_cta - 1) / per_cta, cap = 1 << 20;
  const int grid = (int)(want < cap ? want : cap);
#define EMBED(DT)                                                                               \
  if (vec && rows_long) embed_long_kernel<DT><<<grid, kEmbedThreads, 0, st>>>(A, per_row);      \
  else if (vec) embed_vec_kernel<DT><<<grid, kEmbedThreads, 0, st>>>(A, per_row);               \
  else if (rows_long) embed_shift_long_kernel<DT><<<grid, kEmbedThreads, 0, st>>>(A, per_row);  \
  else embed_shift_kernel<DT><<<grid, kEmbedThreads, 0, st>>>(A, per_row)
  if (dtype == GLS_BF16) {
    EMBED(kBF16);
  } else {
    EMBED(kF32);
  }
#undef EMBED
  return cudaGetLastError() == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

}  // extern "C"

namespace gls {

struct EmbedGradPlan {
  int bits, passes, tiles, per_range, ranges;
  bool small;                  // a cluster sorts, and the CTAs that write zeros look through the tokens
  size_t off_key[2], off_pos[2], off_heads, off_sum, off_cnt, off_touched, off_counters, off_partial, total;
  size_t zero_from, zero_bytes;  // what has to be zero at the start (counts of later passes, touched, counters)
};
static bool embed_grad_sizes_ok(int64_t N, int64_t V, int64_t D) {
  return N >= 0 && N < (1LL << 30) && V > 0 && V < (1LL << 31) - 1 && D > 0 && D < (1LL << 31);
}
// CTAs that write zeros beside a cluster that sorts (one per SM: the sort takes an SM's shared memory)
constexpr int kZeroCtas = 140;
// places of a partial: the columns, and up to seven before them where rows start off 16-byte boundaries
static long long partial_places(int64_t D, bool vec) { return vec ? D : (D + 7 + kEgCols - 1) / kEgCols * kEgCols; }
static EmbedGradPlan embed_grad_plan(int64_t N, int64_t V, int64_t D) {
  EmbedGradPlan p;
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;  // keys 0 .. V
  p.small = N <= kClSortMost && V <= (long long)kZeroCtas * kZeroRows;
  const int most = p.small ? kClSortMaxBits : kSortMaxBits;
  p.passes = (bits + most - 1) / most;
  p.bits = (bits + p.passes - 1) / p.passes;
  const int tile = p.small ? kClSortTile : kSortTile;
  p.tiles = (int)((N + tile - 1) / tile);
  if (p.tiles < 1) p.tiles = 1;
  // as many ranges as fill the machine a few times over, no more: a range's ends cost a partial each
  p.per_range = 8;
  while (p.per_range < kEgMaxRange && N / p.per_range > 2048) p.per_range *= 2;
  p.ranges = (int)((N + p.per_range - 1) / p.per_range);
  size_t at = 0;
  for (int i = 0; i < 2; ++i) {
    p.off_key[i] = at;
    at += up256((size_t)N * 4);
    p.off_pos[i] = at;
    at += up256((size_t)N * 4);
  }
  p.off_heads = at;
  at += up256((size_t)p.ranges * 2 * sizeof(int4));
  p.off_sum = at;
  at += up256((size_t)p.passes * kSortBins * 4);
  p.off_cnt = at;
  const size_t first = (size_t)p.tiles * kSortBins * 4;
  at += up256((size_t)p.passes * first);
  p.off_touched = at;
  at += up256((size_t)((V + 31) / 32) * 4);
  p.off_counters = at;
  at += 256;
  p.zero_from = p.off_cnt + first;
  p.zero_bytes = at - p.zero_from;
  p.off_partial = at;
  at += up256((size_t)p.ranges * 2 * (size_t)partial_places(D, false) * 4);
  p.total = at;
  return p;
}

// Launches a kernel as a programmatic dependent of the one before it in the stream.
template <class... P, class... Args>
static cudaError_t launch_after(void (*kernel)(P...), unsigned grid, int block, cudaStream_t st, Args... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

static cudaError_t launch_cluster_sort(const SortArgs& S, int* counters, int ctas, unsigned grid, const ZeroShare& h,
                                       cudaStream_t st) {
  const int smem = (int)sizeof(ClSortShared);
  const cudaError_t err = cudaFuncSetAttribute(embed_sort_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kClSortThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, embed_sort_cluster_kernel, S, counters, ctas, h);
}

// Deals rows of zeros to the launches.
struct ZeroDeal {
  long long next, V, row_bytes;
  ZeroShare take(long long rows, int from, int each) {
    ZeroShare h;
    h.from = from;
    h.each = each;
    h.first = next;
    next = rows < V - next ? next + rows : V;
    h.last = next;
    return h;
  }
  // rows that about `bytes` make up
  long long worth(double bytes) const { return (long long)(bytes / (double)row_bytes); }
  static unsigned ctas(const ZeroShare& h) { return (unsigned)(h.from + (h.last - h.first + h.each - 1) / h.each); }
};

template <int DT, int DTO, bool VEC>
static cudaError_t launch_embed_grad(const EmbedGradArgs& A, ZeroDeal& deal, int threads, int each, cudaStream_t st) {
  const int n_sum = A.ranges * A.slabs;
  // the join takes some 10 us of which little is spent on memory
  const long long rest = deal.V - deal.next, last = A.ranges > 1 ? (deal.worth(48e6) < rest / 2 ? deal.worth(48e6) : rest / 2) : 0;
  const ZeroShare h = deal.take(rest - last, n_sum, each);
  cudaError_t err = launch_after(embed_grad_kernel<DT, DTO, VEC>, ZeroDeal::ctas(h), threads, st, A, h);
  if (err != cudaSuccess || A.ranges < 2) return err;
  const long long tiles = (A.partial_stride + 4 * kEgThreads - 1) / (4 * kEgThreads) * A.ranges;
  const long long cap = (long long)sm_count() * 8;
  const ZeroShare j = deal.take(deal.V, (int)(tiles < cap ? tiles : cap), each);
  return launch_after(embed_join_kernel<DTO>, ZeroDeal::ctas(j), kEgThreads, st, A, j);
}

}  // namespace gls

extern "C" {

size_t gls_embed_tokens_backward_workspace_bytes(int64_t N, int64_t V, int64_t D) {
  return embed_grad_sizes_ok(N, V, D) ? embed_grad_plan(N, V, D).total : 0;
}

int gls_embed_tokens_backward(const void* grad_out, int dtype, int64_t grad_out_stride, const int32_t* tokens,
                              int64_t N, int64_t V, int64_t D, float scale, void* grad_table, int grad_dtype,
                              int64_t grad_table_stride, uint32_t flags, void* workspace, size_t workspace_bytes,
                              uint32_t* device_status, void* stream) {
  if (!embed_grad_sizes_ok(N, V, D) || !std::isfinite(scale) || (flags & ~GLS_EMBED_ACCUMULATE) || !grad_table ||
      (V > 1 && grad_table_stride < D))
    return GLS_ERR_INVALID_ARG;
  if ((dtype != GLS_F32 && dtype != GLS_BF16) || (grad_dtype != GLS_F32 && grad_dtype != GLS_BF16) ||
      (dtype == GLS_F32 && grad_dtype == GLS_BF16))
    return GLS_ERR_UNSUPPORTED;
  const bool accumulate = (flags & GLS_EMBED_ACCUMULATE) != 0;
  if (N > 0 && (!grad_out || !tokens || (N > 1 && grad_out_stride < D))) return GLS_ERR_INVALID_ARG;
  const int es = dtype == GLS_F32 ? 4 : 2, eso = grad_dtype == GLS_F32 ? 4 : 2;
  if ((uintptr_t)grad_out % es || (uintptr_t)grad_table % eso) return GLS_ERR_MISALIGNED;
  cudaStream_t st = (cudaStream_t)stream;
  if (N == 0) {
    if (accumulate) return GLS_OK;
    return cudaMemset2DAsync(grad_table, (size_t)(V > 1 ? grad_table_stride : D) * eso, 0, (size_t)D * eso, (size_t)V, st) ==
                   cudaSuccess
               ? GLS_OK
               : GLS_ERR_CUDA;
  }
  const EmbedGradPlan P = embed_grad_plan(N, V, D);
  if (!workspace || workspace_bytes < P.total) return GLS_ERR_WORKSPACE;
  if ((uintptr_t)workspace % 16) return GLS_ERR_MISALIGNED;
  // zeros are written before the gradient's rows are read
  if (rows_meet(grad_out, N, grad_out_stride * es, D * es, grad_table, V, grad_table_stride * eso, D * eso))
    return GLS_ERR_INVALID_ARG;
  char* ws = (char*)workspace;
  const bool vec = D % kEgCols == 0 && grad_out_stride * es % 16 == 0 && grad_table_stride * eso % 16 == 0 &&
                   (uintptr_t)grad_out % 16 == 0 && (uintptr_t)grad_table % 16 == 0;
  const long long places = partial_places(D, vec), per_thread = places / kEgCols;
  const int threads = (int)(per_thread < kEgThreads ? (per_thread + 31) / 32 * 32 : kEgThreads);
  const long long slabs = (places + (long long)threads * kEgCols - 1) / ((long long)threads * kEgCols);
  if (slabs * P.ranges > (1LL << 30)) return GLS_ERR_UNSUPPORTED;
  ZeroArgs Z;
  Z.out = (char*)grad_table;
  Z.out_stride = grad_table_stride;
  Z.V = (int)V;
  Z.D = D;
  Z.es = eso;
  const bool even = D * eso % 16 == 0 && grad_table_stride * eso % 16 == 0 && (uintptr_t)grad_table % 16 == 0;
  Z.units = even ? D * eso / 16 : row_pieces(D * eso, eso);
  Z.how = P.small ? kZeroByTokens : kZeroByBits;
  Z.touched = (const uint32_t*)(ws + P.off_touched);
  Z.tokens = tokens;
  Z.keys = (const int32_t*)(ws + P.off_key[(P.passes - 1) & 1]);
  Z.N = (int)N;
  ZeroDeal deal = {accumulate ? (long long)V : 0, (long long)V, (long long)D * eso};
  // Rows per CTA that writes zeros: some 64 KB each, and no more than 2^20 CTAs.  Behind a cluster that
  // sorts, a CTA first has to find out which of its rows to leave: among few tokens it looks through all
  // of them, which lets it start beside the sort (1184 CTAs, eight per SM), among many it waits and finds
  // its own among the sorted ones (256 KB of rows each).
  const bool by_tokens = P.small && N <= 8192;
  long long each = by_tokens ? (V + 1183) / 1184 : (P.small ? 262144 : 65536) / deal.row_bytes;
  if (each < 1) each = 1;
  if (each < (V >> 20) + 1) each = (V >> 20) + 1;
  if (P.small && each > kZeroRows) each = kZeroRows;
  SortArgs S;
  S.tokens = tokens;
  S.N = (int)N;
  S.V = (int)V;
  S.bits = P.bits;
  S.passes = P.passes;
  S.tiles = P.tiles;
  S.cnt = (uint32_t*)(ws + P.off_cnt);
  S.sum = (uint32_t*)(ws + P.off_sum);
  S.touched = accumulate ? nullptr : (uint32_t*)(ws + P.off_touched);
  for (int i = 0; i < 2; ++i) {
    S.key[i] = (int32_t*)(ws + P.off_key[i]);
    S.pos[i] = (int32_t*)(ws + P.off_pos[i]);
  }
  S.status = device_status;
  S.zero = Z;
  int* const counters = (int*)(ws + P.off_counters);
  if (P.small) {
    int ctas = 1;
    while (ctas < P.tiles) ctas *= 2;
    // the sort takes 10 us and more
    ZeroShare h = deal.take(deal.worth(64e6), ctas, 1);
    h.each = (int)((h.last - h.first + kZeroCtas - 1) / kZeroCtas);
    if (h.each < 1) h.each = 1;
    const unsigned grid = (ZeroDeal::ctas(h) + ctas - 1) / ctas * ctas;  // whole clusters
    if (launch_cluster_sort(S, counters, ctas, grid, h, st) != cudaSuccess) return GLS_ERR_CUDA;
  } else {
    if (cudaMemsetAsync(ws + P.zero_from, 0, P.zero_bytes, st) != cudaSuccess) return GLS_ERR_CUDA;
    embed_sort_count_kernel<<<P.tiles, kSortThreads, 0, st>>>(S);
    for (int pass = 0; pass < P.passes; ++pass) {
      if (P.tiles > kSortFewTiles &&
          launch_after(embed_sort_scan_kernel, kSortBins / 32, 32 * kScanWarps, st, S, pass) != cudaSuccess)
        return GLS_ERR_CUDA;
      const ZeroShare h = deal.take(deal.worth(64e6), P.tiles, (int)each);  // a pass takes some 10 us
      if (launch_after(embed_sort_pass_kernel, ZeroDeal::ctas(h), kSortThreads, st, S, pass, h) != cudaSuccess)
        return GLS_ERR_CUDA;
    }
  }
  if (cudaGetLastError() != cudaSuccess) return GLS_ERR_CUDA;
  EmbedGradArgs A;
  A.g = (const char*)grad_out;
  A.g_stride = grad_out_stride;
  A.out = (char*)grad_table;
  A.out_stride = grad_table_stride;
  A.key = S.key[(P.passes - 1) & 1];
  A.pos = S.pos[(P.passes - 1) & 1];
  A.partial = (float*)(ws + P.off_partial);
  A.counters = counters;
  A.heads = (int4*)(ws + P.off_heads);
  A.N = (int)N;
  A.V = (int)V;
  A.D = D;
  A.per_range = P.per_range;
  A.ranges = P.ranges;
  A.accumulate = accumulate ? 1 : 0;
  A.scale = scale;
  A.slabs = (int)slabs;
  A.partial_stride = places;
  A.zero = Z;
  if (P.small && !by_tokens) A.zero.how = kZeroByKeys;
  cudaError_t err;
#define EMBED_GRAD(DT, DTO) \
  err = vec ? launch_embed_grad<DT, DTO, true>(A, deal, threads, (int)each, st) \
            : launch_embed_grad<DT, DTO, false>(A, deal, threads, (int)each, st)
  if (dtype == GLS_F32) EMBED_GRAD(kF32, kF32);
  else if (grad_dtype == GLS_F32) EMBED_GRAD(kBF16, kF32);
  else EMBED_GRAD(kBF16, kBF16);
#undef EMBED_GRAD
  return err == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

}  // extern "C"
