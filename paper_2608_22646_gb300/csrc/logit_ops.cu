// Host side of the operators on rows of logits declared in include/cai.h:
// argument checks and launches of the sampling, record and distillation kernels.
// They keep no state and need no workspace.
#include <cuda_runtime.h>

#include <cmath>
#include <mutex>

#include "cai.h"
#include "distill.cuh"
#include "row_ops.cuh"
#include "sample.cuh"

using namespace cai;

namespace {

constexpr int kMaxDevices = 64;
constexpr int kRowMaxV = 262144;

bool on_this_device(const void* p, int dev) {
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return (a.type == cudaMemoryTypeDevice || a.type == cudaMemoryTypeManaged) && a.device == dev;
}

struct RowDevice {
  int dev = 0;
  int sms = 0;
  bool ready = false;
  // Shared memory: what a launch may ask for, and what the kernels have already.
  size_t limit[3] = {}, fixed[3] = {};
};
enum { kSample, kTop, kDistill };
std::mutex g_row_mutex;
RowDevice g_row[kMaxDevices];

template <typename K>
bool open_smem(K* kernel, int optin, RowDevice* d, int which) {
  cudaFuncAttributes a{};
  if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess) return false;
  const size_t n = static_cast<size_t>(optin) - a.sharedSizeBytes;
  if (d->limit[which] == 0 || n < d->limit[which]) {
    d->limit[which] = n;
    d->fixed[which] = a.sharedSizeBytes;
  }
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(n)) == cudaSuccess &&
         cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                              cudaSharedmemCarveoutMaxShared) == cudaSuccess;
}

// The current device, whose kernels' shared-memory limits are set on first use.
int row_device(RowDevice** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  RowDevice& d = g_row[dev];
  std::lock_guard<std::mutex> lock(g_row_mutex);
  if (!d.ready) {
    int major = 0, minor = 0, optin = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
      cudaGetLastError();
      return CAI_ERR_CUDA;
    }
    if (major != 10 || minor != 3) return CAI_ERR_UNSUPPORTED;
    using bf16 = __nv_bfloat16;
    if (cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess ||
        !open_smem(sample_rows_kernel<float, true>, optin, &d, kSample) ||
        !open_smem(sample_rows_kernel<float, false>, optin, &d, kSample) ||
        !open_smem(sample_rows_kernel<bf16, true>, optin, &d, kSample) ||
        !open_smem(sample_rows_kernel<bf16, false>, optin, &d, kSample) ||
        !open_smem(top_rows_kernel<float, true>, optin, &d, kTop) ||
        !open_smem(top_rows_kernel<float, false>, optin, &d, kTop) ||
        !open_smem(top_rows_kernel<bf16, true>, optin, &d, kTop) ||
        !open_smem(top_rows_kernel<bf16, false>, optin, &d, kTop) ||
        !open_smem(distill_kernel<float, true>, optin, &d, kDistill) ||
        !open_smem(distill_kernel<float, false>, optin, &d, kDistill) ||
        !open_smem(distill_kernel<bf16, true>, optin, &d, kDistill) ||
        !open_smem(distill_kernel<bf16, false>, optin, &d, kDistill)) {
      cudaGetLastError();
      return CAI_ERR_CUDA;
    }
    d.dev = dev;
    d.ready = true;
  }
  *out = &d;
  return CAI_OK;
}

int elem_bytes(int dtype) { return dtype == CAI_BF16 ? 2 : dtype == CAI_F32 ? 4 : 0; }

// Sizes and strides that every operator on rows shares.
int check_rows(const void* p, int32_t dtype, int64_t ld, int32_t M, int32_t V) {
  const int e = elem_bytes(dtype);
  if (!e || (!p && M != 0)) return CAI_ERR_ARG;  // no rows, no buffers
  if (M < 0 || V < 1 || V > kRowMaxV || M > (INT32_MAX / kRowMaxCluster)) return CAI_ERR_SHAPE;
  if (ld < V || reinterpret_cast<uintptr_t>(p) % e != 0) return CAI_ERR_ARG;
  return CAI_OK;
}

// Positive, and log2(e) / t a number in 32 bits, as t is.
bool is_temperature(float t) {
  return t > 0.0f && std::isfinite(t) && std::isfinite(kRowLog2e / t);
}

bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// A cluster of CTAs, or one alone, for every row.  `extra`: dynamic shared memory
// beside the slice, for that many elements of it.
template <typename P>
int launch_rows(void (*cluster)(P, int), void (*alone)(P, int), const P& p, int M, int V, int elem,
                const RowDevice& d, int which, void* stream, size_t (*extra)(int)) {
  const RowPlan plan =
      row_plan(M, V, elem, d.sms, d.limit[which], d.fixed[which], extra);
  const bool split = plan.ctas > 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(split ? M * plan.ctas : M));
  cfg.blockDim = dim3(plan.threads);
  cfg.dynamicSmemBytes = plan.smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = split ? plan.ctas : 1;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = split ? 1 : 0;
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (cudaLaunchKernelEx(&cfg, split ? cluster : alone, p, split ? plan.ctas : plan.room) !=
      cudaSuccess) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  return CAI_OK;
}

size_t nothing(int) { return 0; }

}  // namespace

extern "C" int cai_sample_rows(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                               const float* temperature, const int32_t* top_k, const float* top_p,
                               const float* min_p, const float* u, int32_t* token, float* prob,
                               void* stream) {
  int r = check_rows(logits, dtype, ld, M, V);
  if (r != CAI_OK || M == 0) return r;
  if (!u || !token || !prob) return CAI_ERR_ARG;
  RowDevice* d = nullptr;
  if ((r = row_device(&d)) != CAI_OK) return r;
  const void* ptrs[] = {logits, temperature, top_k, top_p, min_p, u, token, prob};
  for (const void* p : ptrs)
    if (p && ((p != logits && !aligned4(p)) || !on_this_device(p, d->dev))) return CAI_ERR_ARG;
  SampleParams p{logits, ld, M, V, temperature, top_k, top_p, min_p, u, token, prob};
  return dtype == CAI_BF16
             ? launch_rows(sample_rows_kernel<__nv_bfloat16, true>,
                           sample_rows_kernel<__nv_bfloat16, false>, p, M, V, 2, *d, kSample, stream, nothing)
             : launch_rows(sample_rows_kernel<float, true>, sample_rows_kernel<float, false>, p, M, V,
                           4, *d, kSample, stream, nothing);
}

extern "C" int cai_top_rows(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                            int32_t K, double temperature, float* values, int32_t* index,
                            float* lse, void* stream) {
  int r = check_rows(logits, dtype, ld, M, V);
  if (r != CAI_OK) return r;
  if (K < 1 || K > kTopMax || K > V) return CAI_ERR_SHAPE;
  const float t = static_cast<float>(temperature);
  if (!is_temperature(t)) return CAI_ERR_ARG;
  if (M == 0) return CAI_OK;
  if (!values || !index || !lse) return CAI_ERR_ARG;
  RowDevice* d = nullptr;
  if ((r = row_device(&d)) != CAI_OK) return r;
  const void* ptrs[] = {logits, values, index, lse};
  for (const void* p : ptrs)
    if ((p != logits && !aligned4(p)) || !on_this_device(p, d->dev)) return CAI_ERR_ARG;
  TopParams p{logits, ld, M, V, K, t, values, index, lse};
  return dtype == CAI_BF16
             ? launch_rows(top_rows_kernel<__nv_bfloat16, true>, top_rows_kernel<__nv_bfloat16, false>,
                           p, M, V, 2, *d, kTop, stream, nothing)
             : launch_rows(top_rows_kernel<float, true>, top_rows_kernel<float, false>, p, M, V, 4,
                           *d, kTop, stream, nothing);
}

namespace {

int distill_call(DistillParams& p, int32_t dtype, int64_t ld_grad, void* stream) {
  int r = check_rows(p.logits, dtype, p.ld, p.M, p.V);
  if (r != CAI_OK) return r;
  const int e = elem_bytes(dtype);
  if (p.K < 1 || p.K > kTopMax) return CAI_ERR_SHAPE;
  if (!is_temperature(p.tau)) return CAI_ERR_ARG;
  if (p.M == 0) return CAI_OK;
  if (!p.top_values || !p.top_index || !p.stats || (!p.loss && (!p.upstream || !p.grad)))
    return CAI_ERR_ARG;
  if (p.grad && (ld_grad < p.V || reinterpret_cast<uintptr_t>(p.grad) % e != 0)) return CAI_ERR_ARG;
  RowDevice* d = nullptr;
  if ((r = row_device(&d)) != CAI_OK) return r;
  const void* ptrs[] = {p.top_values, p.top_index, p.top_lse, p.weight,
                        p.loss,       p.stats,     p.upstream};
  for (const void* q : ptrs)
    if (q && (!aligned4(q) || !on_this_device(q, d->dev))) return CAI_ERR_ARG;
  if (!on_this_device(p.logits, d->dev) || (p.grad && !on_this_device(p.grad, d->dev)))
    return CAI_ERR_ARG;
  p.ld_grad = ld_grad;
  return dtype == CAI_BF16
             ? launch_rows(distill_kernel<__nv_bfloat16, true>, distill_kernel<__nv_bfloat16, false>, p,
                           p.M, p.V, 2, *d, kDistill, stream, bitmap_bytes)
             : launch_rows(distill_kernel<float, true>, distill_kernel<float, false>, p, p.M, p.V, 4,
                           *d, kDistill, stream, bitmap_bytes);
}

}  // namespace

extern "C" int cai_distill_loss(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                                int32_t K, const float* top_values, const int32_t* top_index,
                                const float* top_lse, double temperature, const float* weight,
                                float* loss, float* stats, void* grad, int64_t ld_grad,
                                void* stream) {
  DistillParams p{logits, ld,   M,     V,       K,    static_cast<float>(temperature), top_values,
                  top_index, top_lse, weight, loss, stats, nullptr, grad, 0};
  return distill_call(p, dtype, ld_grad, stream);
}

extern "C" int cai_distill_backward(const void* logits, int32_t dtype, int64_t ld, int32_t M,
                                    int32_t V, int32_t K, const float* top_values,
                                    const int32_t* top_index, const float* top_lse,
                                    double temperature, const float* weight, const float* stats,
                                    const float* grad_loss, void* grad, int64_t ld_grad,
                                    void* stream) {
  DistillParams p{logits, ld,   M,       V,    K,       static_cast<float>(temperature),
                  top_values, top_index, top_lse, weight, nullptr,
                  const_cast<float*>(stats), grad_loss, grad, 0};
  return distill_call(p, dtype, ld_grad, stream);
}
