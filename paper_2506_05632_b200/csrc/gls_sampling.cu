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
  if (A.V <= 8192) return launch_sample<DT, 128>(A, rows, 1, st);
  // More rows than SMs: four small CTAs an SM hide one another's waits, a large one is done sooner with a row that has to be
  // summed in 64 bits.  128256 bf16 tokens, the same rows, small / large: top-k 50 and top-p 0.9, 200 rows 33 / 40 us,
  // 592 59 / 88, 888 90 / 126; min-p 0.05, 592 46 / 63; top-k 1000 alone 592 170 / 185, but 296 115 / 90; where rows may be
  // summed, settings of their own, 200 rows 192-220 / 110-129, 512 222-236 / 139-193, 888 262-319 / 225-241, 2048 409-435 /
  // 436-470; nothing restricted, 592 115-132 / 81-113, 888 135 / 123-141, 2048 195-200 / 240-262.
  if (rows * 2 > sms)
    return rows > (may_sum(A) ? 4 : 1) * (long long)sms ? launch_sample<DT, 256>(A, rows, 1, st) : launch_sample<DT, 512>(A, rows, 1, st);
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
