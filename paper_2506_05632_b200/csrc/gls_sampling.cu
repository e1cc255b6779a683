// gls_sampling.cu -- C ABI of independent sampling by temperature, top-k, top-p and min-p (see include/gls.h).
#include <cmath>

#include "../../include/gls.h"
#include "gls_host.cuh"
#include "gls_sample.cuh"

namespace gls {

static_assert(kSampleBadSetting == GLS_DEV_BAD_SETTING, "header");

static SampleSetting setting(const void* rows, const int64_t* stride, float value, int ivalue) {
  SampleSetting s;
  s.rows = rows;
  s.sb = stride[0], s.sk = stride[1], s.sj = stride[2];
  s.value = value;
  s.ivalue = ivalue;
  return s;
}

template <int DT, int THREADS>
static cudaError_t launch_sample(SampleArgs& A, long long rows, int ctas, cudaStream_t st) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * ctas));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = ctas > 1 ? 1 : 0;
  cfg.dynamicSmemBytes = sizeof(SampleShared<DT, THREADS>);
  const cudaError_t err = cudaFuncSetAttribute(sample_kernel<DT, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
  if (err != cudaSuccess) return err;
  return cudaLaunchKernelEx(&cfg, sample_kernel<DT, THREADS>, A);
}

// whether a row may need a total over all its tokens: neither all rows have a top-k, nor all a min-p without a top-p
static bool may_sum(const SampleArgs& A) {
  const bool top_k = !A.top_k.rows && A.top_k.ivalue > 0 && A.top_k.ivalue < A.V, greedy = !A.inv_temp.rows && std::isinf(A.inv_temp.value);
  const bool min_p = !A.min_p.rows && A.min_p.value > 0.f && !A.top_p.rows && A.top_p.value >= 1.f;
  return !top_k && !greedy && !min_p;
}

template <int DT>
static cudaError_t launch_sample_rows(SampleArgs& A, long long rows, cudaStream_t st) {
  // as few positions per chunk as leave the row no more chunks than there is room for
  A.shift = 0;
  while ((((long long)A.V + 7 + (256LL << A.shift) - 1) >> (8 + A.shift)) > kSampleChunks) ++A.shift;
  // few rows: several CTAs sweep one, so that most SMs have a share of it
  const int sms = sm_count();
  // One CTA a row: four small ones an SM hide one another's waits, a large one is done sooner with a row that has to be summed in 64
  // bits or has many tokens to choose among.  Rows without such work take the small one beyond one row an SM, others once the rest of
  // the grid hides theirs, the later the longer they are: beyond one row an SM per 48 KB of a row where nothing restricts them, per
  // 32 KB with top-p or a large top-k, per 16 KB with settings of their own.  bf16 rows of 32000 / 152064 tokens, small : large, us:
  // min-p 0.05, 200 rows 19 : 24 / 30 : 34, 1184 42 : 80 / 96 : 129; nothing, 200 rows 18 : 24 / 73 : 56, 592 38 : 48 / 136 : 108,
  // 1776 76 : 144 / 213 : 252; p = 0.9, 200 rows 68 : 66 / 223 : 130, 592 73 : 110 / 303 : 249, 1776 199 : 313 / 622 : 670; top-k
  // 1000, 200 rows 86 : 88 / 110 : 100, 592 115 : 172 / 194 : 207 (fp32 128256: 395 : 222); settings of their own, 296 rows
  // 110 : 92 / 282 : 175, 592 120 : 134 / 356 : 260, 2368 378 : 422 / 644 : 622.
  const bool sums = may_sum(A), many = !A.top_k.rows && A.top_k.ivalue > 256 && A.top_k.ivalue < A.V;
  const bool own = A.inv_temp.rows || A.top_k.rows || A.top_p.rows || A.min_p.rows;
  const bool top_p = A.top_p.rows || A.top_p.value < 1.f;
  if (A.V <= 8192) {
    // A few KB a row: eight CTAs of 128 threads an SM once four of 256 leave rows waiting, where there is little to do for one.
    // bf16 rows of 1000 / 8192 tokens, 128 : 256 threads: nothing, 592 rows 18 : 17 / 21 : 19, 740 18 : 25 / 23 : 25; top-k 1, 740 rows
    // 18 : 28 / 18 : 26; p = 0.9, 888 rows 55 : 50 / 66 : 56; settings of their own, 740 rows 64 : 68 / 97 : 84.
    return rows > 4LL * sms && !many && !(sums && (own || top_p)) ? launch_sample<DT, 128>(A, rows, 1, st) : launch_sample<DT, 256>(A, rows, 1, st);
  }
  if (rows * 2 > sms) {
    const long long bytes = (long long)A.V * SampleRow<DT>::ES, unit = many ? 32768 : own ? 16384 : top_p ? 32768 : 49152;
    const bool large = rows <= sms || ((sums || many) && rows * unit <= bytes * sms);
    return large ? launch_sample<DT, 512>(A, rows, 1, st) : launch_sample<DT, 256>(A, rows, 1, st);
  }
  int ctas = 2;
  while (ctas < 8 && rows * ctas * 2 <= sms && A.V > 8192 * ctas) ctas *= 2;
  return launch_sample<DT, 512>(A, rows, ctas, st);
}

}  // namespace gls

extern "C" int gls_sample_tokens(const gls_rows_t* logits, int B, int K, int J, int64_t V, const gls_sampling_t* s,
                                 const float* uniforms, int32_t* out_tokens, float* out_logprobs, uint32_t* device_status,
                                 void* stream) {
  using namespace gls;
  if (B <= 0 || K <= 0 || K > GLS_MAX_K || J <= 0 || V <= 0 || V >= (1LL << 31) - 65536 ||
      (long long)B * K * J >= (1LL << 31) / 64 || !logits || !logits->data || !s || !uniforms || !out_tokens)
    return GLS_ERR_INVALID_ARG;
  if (logits->dtype != GLS_F32 && logits->dtype != GLS_BF16) return GLS_ERR_UNSUPPORTED;
  if ((uintptr_t)logits->data % (logits->dtype == GLS_F32 ? 4 : 2)) return GLS_ERR_MISALIGNED;
  if (!s->inv_temp_rows) {
    if (!(s->inv_temp > 0.f)) return GLS_ERR_INVALID_ARG;
    if (s->inv_temp < 1e-20f || (s->inv_temp > 1e20f && !std::isinf(s->inv_temp))) return GLS_ERR_UNSUPPORTED;
  }
  if (!s->top_p_rows && !(s->top_p > 0.f)) return GLS_ERR_INVALID_ARG;
  if (!s->min_p_rows && !(s->min_p >= 0.f && s->min_p <= 1.f)) return GLS_ERR_INVALID_ARG;
  SampleArgs A;
  A.data = logits->data;
  A.sb = logits->stride_b, A.sk = logits->stride_k, A.sj = logits->stride_j;
  A.K = K, A.J = J, A.V = (int)V;
  A.inv_temp = setting(s->inv_temp_rows, s->inv_temp_stride, s->inv_temp, 0);
  A.top_k = setting(s->top_k_rows, s->top_k_stride, 0.f, s->top_k);
  A.top_p = setting(s->top_p_rows, s->top_p_stride, s->top_p, 0);
  A.min_p = setting(s->min_p_rows, s->min_p_stride, s->min_p, 0);
  A.u = uniforms;
  A.tokens = out_tokens;
  A.logprobs = out_logprobs;
  A.status = device_status;
  const long long rows = (long long)B * K * J;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = logits->dtype == GLS_F32 ? launch_sample_rows<kF32>(A, rows, st) : launch_sample_rows<kBF16>(A, rows, st);
  return err == cudaSuccess ? GLS_OK : GLS_ERR_CUDA;
}
