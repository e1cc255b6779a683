// gls_int4.cu -- C ABI of 4-bit tables (see include/gls.h): made from weights, read by token, multiplied with
// hidden states.
#include <cmath>

#include "../../include/gls.h"
#include "gls_host.cuh"
#include "gls_head_wide.cuh"

namespace gls {

static bool float_type(int dtype) { return dtype == GLS_F32 || dtype == GLS_BF16; }

static int table_of(const gls_int4_table_t* t, Int4Table* out) {
  if (!t || !t->codes || !t->scales || t->V <= 0 || t->V >= (1LL << 31) - 65536 || t->D <= 0) return GLS_ERR_INVALID_ARG;
  if (t->group != 32 && t->group != 64 && t->group != 128) return GLS_ERR_UNSUPPORTED;
  if (!float_type(t->scale_dtype) || t->D > 32768) return GLS_ERR_UNSUPPORTED;
  const int64_t G = (t->D + t->group - 1) / t->group;
  if (t->V > 1 && (t->code_stride < (t->D + 31) / 32 * 16 || t->scale_stride < G || (t->zeros && t->zero_stride < G)))
    return GLS_ERR_INVALID_ARG;
  if ((uintptr_t)t->codes % 16 || (t->V > 1 && t->code_stride % 16) || (uintptr_t)t->scales % (t->scale_dtype == GLS_F32 ? 4 : 2))
    return GLS_ERR_MISALIGNED;
  out->codes = t->codes;
  out->code_stride = t->code_stride;
  out->scales = t->scales;
  out->scale_stride = t->scale_stride;
  out->zeros = t->zeros;
  out->zero_stride = t->zero_stride;
  out->V = t->V;
  out->D = t->D;
  out->G = (int)G;
  out->log_group = t->group == 32 ? 5 : t->group == 64 ? 6 : 7;
  out->scale_bf16 = t->scale_dtype == GLS_BF16;
  return GLS_OK;
}

// whether rows of `len` bytes written from p lie in the table's memory
static bool meets_table(const void* p, int64_t n, int64_t pitch, int64_t len, const Int4Table& T) {
  const int64_t ss = T.scale_bf16 ? 2 : 4;
  return rows_meet(p, n, pitch, len, T.codes, T.V, T.code_stride, (T.D + 1) / 2) ||
         rows_meet(p, n, pitch, len, T.scales, T.V, T.scale_stride * ss, T.G * ss) ||
         (T.zeros && rows_meet(p, n, pitch, len, T.zeros, T.V, T.zero_stride, T.G));
}

// threads per row, a power of two that leaves few idle and holds whole groups; CTAs for that many rows
static int lanes_for(long long units, int least) {
  int n = least;
  while (n < units && n < kInt4Threads) n *= 2;
  return n;
}
static unsigned ctas_for(long long rows, int lanes) {
  const long long per = kInt4Threads / lanes, n = (rows + per - 1) / per, cap = (long long)sm_count() * 32;
  return (unsigned)(n < cap ? n : cap);
}

constexpr int kHeadShared = 227 * 1024;  // at most per CTA

// shared memory per hidden state
static long long head_column_bytes(int parts, int chunks, int uc) { return (long long)parts * ((chunks + uc - 1) / uc) * uc * 256; }

// A map of rows x columns, copied in boxes of `rows` rows by `cols` columns.
static bool box_map(CUtensorMapDataType type, void* data, long long columns, long long rows, long long pitch_bytes, int box_columns,
                    int box_rows, CUtensorMapSwizzle swizzle, CUtensorMap* map) {
  typedef decltype(&cuTensorMapEncodeTiled) Encode;
  static std::atomic<Encode> found{nullptr};
  Encode encode = found.load(std::memory_order_relaxed);
  if (!encode) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess || !p) {
      (void)cudaGetLastError();
      return false;
    }
    encode = (Encode)p;
    found.store(encode, std::memory_order_relaxed);
  }
  const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)pitch_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)box_columns, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encode(map, type, 2, data, dims, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The codes as bytes [V][ceil(D / 32) * 16]
static bool codes_map(const Int4Table& T, int rows, CUtensorMapSwizzle swizzle, CUtensorMap* map) {
  const long long row = (T.D + 31) / 32 * 16;
  return box_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, T.codes, row, T.V, T.V > 1 ? T.code_stride : row, 64, rows, swizzle, map);
}

template <int GPC, int PARTS, int UC>
static cudaError_t launch_head_unit(HeadArgs& A, const CUtensorMap& codes, int cols, int warps, cudaStream_t st) {
  A.cols = cols;
  const Int4Table& T = A.T;
  // a lane's scales are half a unit's
  const int ss = T.scale_bf16 ? 2 : 4, per = GPC * UC / 2, align = per * ss < 16 ? per * ss : 16;
  A.vec = (uintptr_t)T.scales % align == 0 && (T.V == 1 || T.scale_stride * ss % align == 0) &&
          (!T.zeros || ((uintptr_t)T.zeros % per == 0 && (T.V == 1 || T.zero_stride % per == 0)));
  void (*const kernel)(HeadArgs, CUtensorMap) = cols == 1   ? head_kernel<GPC, PARTS, 1, UC>
                                                : cols == 2 ? head_kernel<GPC, PARTS, 2, UC>
                                                            : head_kernel<GPC, PARTS, 0, UC>;
  const int smem = (int)(HeadLayout::fixed(GPC, UC, warps) + head_column_bytes(PARTS, A.chunks, UC) * cols);
  // the same for every call: another thread's may come between this and the launch
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadShared);
  if (err != cudaSuccess) return err;
  dim3 grid((unsigned)(A.tiles < sm_count() ? A.tiles : sm_count()), (unsigned)((A.N + cols - 1) / cols));
  kernel<<<grid, 32 * warps, smem, st>>>(A, codes);
  return cudaGetLastError();
}

// As many hidden states per pass as shared memory holds, up to 8; units of four chunks (half the work per unit beside the
// products) where that takes none of them away and a row has that many chunks, otherwise of two.
template <int GPC, int PARTS>
static cudaError_t launch_head(HeadArgs& A, const CUtensorMap& codes, cudaStream_t st) {
  const long long most = kHeadShared, want = A.N < 8 ? A.N : 8;
  if (A.chunks >= 4 && (most - HeadLayout::fixed(GPC, 4, kHeadWarps)) / head_column_bytes(PARTS, A.chunks, 4) >= want)
    return launch_head_unit<GPC, PARTS, 4>(A, codes, (int)want, kHeadWarps, st);
  int warps = kHeadWarps;
  long long cols;
  while ((cols = (most - HeadLayout::fixed(GPC, 2, warps)) / head_column_bytes(PARTS, A.chunks, 2)) < 1) warps /= 2;  // D <= 32768: two have room
  return launch_head_unit<GPC, PARTS, 2>(A, codes, (int)(cols < want ? cols : want), warps, st);
}

// Whether N hidden states take the kernel for many of them: beyond 8, or where shared memory holds so few that the other one
// would take more than two passes over the table (152064 x 4096, groups of 128, 1 .. 8 bf16 hidden states by
// the other one 78 .. 100 us, 9 .. 64 by this one 147 .. 190; 8 fp32 ones 233 in two passes and 209).
static bool head_is_wide(long long N, int parts, long long D) {
  const int chunks = (int)((D + 127) / 128);
  return N > 8 || N * head_column_bytes(parts, chunks, 2) > 2 * (kHeadShared - HeadLayout::fixed(4, 2, kHeadWarps));
}
// How: passes of equal size, 16 .. 64 hidden states at a time.
struct WidePlan {
  int passes, nb;  // nb: 16 hidden states each per pass
  explicit WidePlan(long long N) : passes((int)((N + 63) / 64)), nb((int)((N + 16 * passes - 1) / (16 * passes))) {}
  size_t bytes(int parts, long long D) const { return (size_t)passes * parts * nb * 16 * (size_t)((D + 127) / 128) * 256; }
};

template <int NB, int GPC, int PARTS>
static cudaError_t launch_wide(const HeadArgs& A, const CUtensorMap& codes, int passes, void* workspace, cudaStream_t st) {
  CUtensorMap hidden;
  const long long columns = A.chunks * 128;
  if (!box_map(CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, workspace, columns, (long long)passes * PARTS * 16 * NB, columns * 2, 64, 16 * NB,
               CU_TENSOR_MAP_SWIZZLE_128B, &hidden))
    return cudaErrorInvalidValue;
  const int smem = WideShared::total(NB, PARTS);
  cudaError_t err = cudaFuncSetAttribute(head_wide_kernel<NB, GPC, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  const long long pairs = (A.T.V + 2 * kWideRows - 1) / (2 * kWideRows), most = sm_count(), words = (long long)passes * 16 * NB * A.chunks * 16;
  head_order_kernel<PARTS><<<(unsigned)(words < 256 * most ? (words + 255) / 256 : most), 256, 0, st>>>(A, 16 * NB, passes, (uint4*)workspace);
  err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pairs < most ? pairs : most), (unsigned)passes);
  cfg.blockDim = dim3(kWideThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, head_wide_kernel<NB, GPC, PARTS>, A, codes, hidden);
}

template <int GPC, int PARTS>
static cudaError_t launch_wide_for(HeadArgs& A, const CUtensorMap& codes, void* workspace, cudaStream_t st) {
  const WidePlan P(A.N);
  const Int4Table& T = A.T;
  // a thread's scales are those of eight groups
  A.vec = (uintptr_t)T.scales % 16 == 0 && (T.V == 1 || T.scale_stride * (T.scale_bf16 ? 2 : 4) % 16 == 0) &&
          (!T.zeros || ((uintptr_t)T.zeros % 8 == 0 && (T.V == 1 || T.zero_stride % 8 == 0)));
  switch (P.nb) {
    case 1: return launch_wide<1, GPC, PARTS>(A, codes, P.passes, workspace, st);
    case 2: return launch_wide<2, GPC, PARTS>(A, codes, P.passes, workspace, st);
    case 3: return launch_wide<3, GPC, PARTS>(A, codes, P.passes, workspace, st);
    default: return launch_wide<4, GPC, PARTS>(A, codes, P.passes, workspace, st);
  }
}

template <int PARTS>
static cudaError_t launch_head_for(HeadArgs& A, void* workspace, cudaStream_t st) {
  CUtensorMap codes;
  const bool wide = head_is_wide(A.N, PARTS, A.T.D);
  if (!codes_map(A.T, wide ? kWideRows : 16, wide ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE, &codes)) return cudaErrorInvalidValue;
  switch (A.T.log_group) {
    case 5: return wide ? launch_wide_for<4, PARTS>(A, codes, workspace, st) : launch_head<4, PARTS>(A, codes, st);
    case 6: return wide ? launch_wide_for<2, PARTS>(A, codes, workspace, st) : launch_head<2, PARTS>(A, codes, st);
    default: return wide ? launch_wide_for<1, PARTS>(A, codes, workspace, st) : launch_head<1, PARTS>(A, codes, st);
  }
}

}  // namespace gls

extern "C" {

int gls_quantize_table(const void* weights, int dtype, int64_t weight_stride, const gls_int4_table_t* table, void* stream) {
  using namespace gls;
  QuantizeArgs A;
  const int rc = table_of(table, &A.T);
  if (rc != GLS_OK) return rc;
  if (!weights || (table->V > 1 && weight_stride < table->D)) return GLS_ERR_INVALID_ARG;
  if (!float_type(dtype)) return GLS_ERR_UNSUPPORTED;
  const int es = dtype == GLS_F32 ? 4 : 2;
  if ((uintptr_t)weights % es) return GLS_ERR_MISALIGNED;
  if (meets_table(weights, table->V, table->V > 1 ? weight_stride * es : table->D * es, table->D * es, A.T)) return GLS_ERR_INVALID_ARG;
  A.w = weights;
  A.stride = weight_stride;
  const bool vec = (uintptr_t)weights % 16 == 0 && (table->V == 1 || weight_stride * es % 16 == 0);
  A.lanes = lanes_for((long long)A.T.G << (A.T.log_group - 4), 1 << (A.T.log_group - 4));
  const unsigned grid = ctas_for(A.T.V, A.lanes);
  cudaStream_t st = (cudaStream_t)stream;
  void (*const kernel)(QuantizeArgs) = dtype == GLS_F32 ? (vec ? quantize_kernel<kF32, true> : quantize_kernel<kF32, false>)
                                                        : (vec ? quantize_kernel<kBF16, true> : quantize_kernel<kBF16, false>);
  kernel<<<grid, kInt4Threads, 0, st>>>(A);
  return cudaGetLastError() == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

size_t gls_head_logits_workspace_bytes(int64_t N, int64_t D, int x_dtype) {
  if (N <= 0 || N > 65535 || D <= 0 || D > 32768 || !gls::float_type(x_dtype)) return 0;
  const int parts = x_dtype == GLS_BF16 ? 1 : 3;
  return gls::head_is_wide(N, parts, D) ? gls::WidePlan(N).bytes(parts, D) : 0;
}

int gls_head_logits(const void* x, int x_dtype, int64_t x_stride, int64_t N, const gls_int4_table_t* table, void* out,
                    int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace gls;
  HeadArgs A;
  const int rc = table_of(table, &A.T);
  if (rc != GLS_OK) return rc;
  if (N < 0 || N > 65535) return GLS_ERR_INVALID_ARG;
  if (!float_type(x_dtype) || !float_type(out_dtype)) return GLS_ERR_UNSUPPORTED;
  if (N == 0) return GLS_OK;
  if (!x || !out || (N > 1 && (x_stride < table->D || out_stride < table->V))) return GLS_ERR_INVALID_ARG;
  if ((uintptr_t)x % (x_dtype == GLS_F32 ? 4 : 2) || (uintptr_t)out % (out_dtype == GLS_F32 ? 4 : 2)) return GLS_ERR_MISALIGNED;
  const int xs = x_dtype == GLS_F32 ? 4 : 2, os = out_dtype == GLS_F32 ? 4 : 2;
  if (meets_table(out, N, N > 1 ? out_stride * os : table->V * os, table->V * os, A.T) ||
      rows_meet(out, N, N > 1 ? out_stride * os : table->V * os, table->V * os, x, N, N > 1 ? x_stride * xs : table->D * xs, table->D * xs))
    return GLS_ERR_INVALID_ARG;
  A.x = (const char*)x;
  A.x_stride = x_stride;
  A.N = (int)N;
  A.out = (char*)out;
  A.out_stride = out_stride;
  A.out_bf16 = out_dtype == GLS_BF16;
  const size_t need = gls_head_logits_workspace_bytes(N, A.T.D, x_dtype);
  if (need) {
    if (!workspace || workspace_bytes < need) return GLS_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 16) return GLS_ERR_MISALIGNED;
    if (rows_meet(out, N, N > 1 ? out_stride * os : table->V * os, table->V * os, workspace, 1, need, need) ||
        rows_meet(x, N, N > 1 ? x_stride * xs : table->D * xs, table->D * xs, workspace, 1, need, need) ||
        meets_table(workspace, 1, need, need, A.T))
      return GLS_ERR_INVALID_ARG;
  }
  A.chunks = (int)((A.T.D + 127) / 128);
  A.tiles = (A.T.V + 15) / 16;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = x_dtype == GLS_BF16 ? launch_head_for<1>(A, workspace, st) : launch_head_for<3>(A, workspace, st);
  return err == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

int gls_embed_tokens_int4(const gls_int4_table_t* table, const int32_t* tokens, int64_t N, float scale, void* out,
                          int out_dtype, int64_t out_stride, uint32_t* device_status, void* stream) {
  using namespace gls;
  EmbedInt4Args A;
  const int rc = table_of(table, &A.T);
  if (rc != GLS_OK) return rc;
  if (N < 0 || N >= (1LL << 31) - 65536 || !std::isfinite(scale)) return GLS_ERR_INVALID_ARG;
  if (!float_type(out_dtype)) return GLS_ERR_UNSUPPORTED;
  if (N == 0) return GLS_OK;
  if (!tokens || !out || (N > 1 && out_stride < table->D)) return GLS_ERR_INVALID_ARG;
  const int es = out_dtype == GLS_F32 ? 4 : 2;
  if ((uintptr_t)out % es) return GLS_ERR_MISALIGNED;
  const int64_t pitch = N > 1 ? out_stride * es : table->D * es;
  if (meets_table(out, N, pitch, table->D * es, A.T) || rows_meet(out, N, pitch, table->D * es, tokens, 1, N * 4, N * 4))
    return GLS_ERR_INVALID_ARG;
  A.tokens = tokens;
  A.N = N;
  A.scale = scale;
  A.out = (char*)out;
  A.out_stride = out_stride;
  // fp32 rows go through shared memory even where they are aligned: a thread's 16 columns are four words there, and a warp's
  // store of every fourth word takes longer (128256 x 4096: 578 us, 434 through shared memory; bf16 260 and 402)
  const bool vec = out_dtype == GLS_BF16 && (uintptr_t)out % 16 == 0 && (N == 1 || out_stride * es % 16 == 0);
  A.status = device_status;
  A.lanes = lanes_for((A.T.D + 15) / 16, 1);
  const unsigned grid = ctas_for(N, A.lanes);
  cudaStream_t st = (cudaStream_t)stream;
  void (*const kernel)(EmbedInt4Args) = out_dtype == GLS_F32 ? embed_int4_kernel<kF32, false>
                                        : vec                ? embed_int4_kernel<kBF16, true>
                                                             : embed_int4_kernel<kBF16, false>;
  kernel<<<grid, kInt4Threads, 0, st>>>(A);
  return cudaGetLastError() == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}

}  // extern "C"
