// Host side of the norms of rows declared in include/cai.h: argument checks and
// launches.  They keep no state; the caller gives the backward call's workspace.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "cai.h"
#include "host_checks.h"
#include "norm.cuh"

using namespace cai;

namespace {

int launched() {
  if (cudaGetLastError() != cudaSuccess) return CAI_ERR_CUDA;
  return CAI_OK;
}

int parts_of(int32_t M, int32_t H) { return norm_plan(M, H).parts; }

int check_norm(const void* x, int32_t dtype, int64_t ld, int32_t M, int32_t H, int32_t kind, int32_t wdtype) {
  const int e = elem_bytes(dtype);
  if (!e || !elem_bytes(wdtype) || (!x && M != 0) || (kind != CAI_NORM_LAYER && kind != CAI_NORM_RMS))
    return CAI_ERR_ARG;
  if (M < 0 || H < 1 || H > kNormMaxH) return CAI_ERR_SHAPE;
  if (ld < H || !aligned_to(x, e)) return CAI_ERR_ARG;
  return CAI_OK;
}

// Rows that are written where others are read: their own place, or none of theirs.
bool may_write(const void* out, int64_t ld_out, const void* in, int64_t ld_in, int e, int32_t M, int32_t H) {
  return (out == in && ld_out == ld_in) || !rows_overlap(out, ld_out, e, in, ld_in, e, M, H);
}

// Lets a kernel use up to `most` bytes of dynamic shared memory on the current device;
// set on first use.
template <auto kernel>
bool open_shared(int dev, int most) {
  static std::atomic<bool> open[kMaxDevices];
  if (open[dev].load(std::memory_order_acquire)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  open[dev].store(true, std::memory_order_release);
  return true;
}

constexpr int kMostShared = 216 * 1024;  // of an SM, for the CTAs on it

// Whether rows and vectors of them may be taken 16 bytes at a time.
bool wide_rows(const void* p, int64_t ld, int H, int e) {
  return aligned_to(p, 16) && ld * e % 16 == 0 && H * e % 16 == 0;
}

// Whether rows of these lie alike from 16-byte boundary to 16-byte boundary; those of
// every eighth row then lie alike, of whatever stride.
bool alike(const void* a, int64_t ld_a, const void* b, int64_t ld_b, int e) {
  return (reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) % 16 == 0 && (ld_a - ld_b) * e % 16 == 0;
}

template <typename T, typename W, bool kWide, int kItems>
void forward_items(const NormParams& p, int warps, int sms, cudaStream_t s) {
  constexpr int kResident = 32;  // warps of an SM
  const int groups = warps > 1 ? 1 : 8;
  const long long want = (static_cast<long long>(p.M) + groups - 1) / groups;
  const long long most = sms * static_cast<long long>(kResident / (groups * warps));
  norm_rows_kernel<T, W, kWide, kItems, false>
      <<<static_cast<unsigned>(std::min(want, most)), groups * warps * 32, 0, s>>>(p, warps);
}

// Weight and bias in shared memory, for CTAs that take many rows: four and more for every
// group of warps.
template <typename T, typename W, bool kWide, int kItems, bool kEdges>
bool forward_staged(const NormParams& p, int items, int dev, int sms, cudaStream_t s) {
  const int warps = (items + 32 * kItems - 1) / (32 * kItems), groups = 16 / warps;
  if (!groups) return false;
  const int cols = kEdges ? staged_cols(p.H + 16 / static_cast<int>(sizeof(T)) - 1) : p.H;
  const size_t smem = 2ull * cols * sizeof(float);
  const int ctas = static_cast<int>(std::min<size_t>(2, kMostShared / smem));  // of an SM
  // (rows that start anywhere: else an element at a time.  2000 of 4099 bf16: 39 us)
  if (kEdges ? p.M < sms * ctas : (!p.weight && !p.bias) || p.M < 4ll * sms * ctas * groups) return false;
  if (!open_shared<norm_rows_kernel<T, W, kWide, kItems, true, kEdges>>(dev, 2 * (kNormMaxH + 16) * sizeof(float))) return false;
  norm_rows_kernel<T, W, kWide, kItems, true, kEdges><<<sms * ctas, groups * warps * 32, smem, s>>>(p, warps);
  return true;
}

// Four rows and more for every unit.  False: fewer, or no room for two rows of each.
template <typename T, typename W, int kElems, int kThreads>
bool forward_ring(const NormParams& p, int dev, int sms, cudaStream_t s) {
  const int span = (p.H + kElems * 32 - 1) / (kElems * 32) * 32, units = kThreads / span;
  const int threads = units * span, row = kThreads * kElems * static_cast<int>(sizeof(T));
  const int ring = units ? std::min(8, kMostShared / row) : 0;
  if (ring < 2 || p.M < 4 * sms * units || !open_shared<norm_ring_kernel<T, W, kElems, kThreads>>(dev, kMostShared))
    return false;
  norm_ring_kernel<T, W, kElems, kThreads><<<sms, threads, ring * row, s>>>(p, span, ring);
  return true;
}

template <typename T, typename W, bool kWide>
void forward(const NormParams& p, int dev, int sms, cudaStream_t s) {
  // Many rows that lie alike: wide ones through rings, others a row to as few warps as hold
  // it, four items to a thread.
  if (kWide || (sms % 8 == 0 && p.H >= 64 && alike(p.x, p.ld, p.out, p.ld_out, sizeof(T)))) {
    constexpr int kN = Item<T, true>::kN, kMore = kWide ? 0 : kN - 1, kHeld = 4;
    constexpr bool bf16 = sizeof(T) == 2;
    if constexpr (kWide)
      if (p.H > 4096 && forward_ring<T, W, bf16 ? 32 : 16, bf16 ? 512 : 768>(p, dev, sms, s)) return;
    if (forward_staged<T, W, true, kHeld, !kWide>(p, (p.H + kMore + kN - 1) / kN, dev, sms, s)) return;
  }
  const int items = p.H / Item<T, kWide>::kN;
  if constexpr (!kWide)  // eight elements to a thread
    if (forward_staged<T, W, false, 8, false>(p, items, dev, sms, s)) return;
  // Else eight items of 16 bytes to a thread (or 16 elements); more warps while rows are
  // so few that they are idle otherwise.
  int warps = 1;
  while (warps < kNormMaxWarps && items > warps * 32 * (kWide ? 8 : 16)) warps *= 2;
  while (warps < kNormMaxWarps && items > warps * 32 && static_cast<long long>(p.M) * warps * 2 <= sms * 16ll) warps *= 2;
  const int each = (items + warps * 32 - 1) / (warps * 32);
  if (each <= 1) return forward_items<T, W, kWide, 1>(p, warps, sms, s);
  if (each <= 2) return forward_items<T, W, kWide, 2>(p, warps, sms, s);
  if (each <= 4) return forward_items<T, W, kWide, 4>(p, warps, sms, s);
  if (each <= 8) return forward_items<T, W, kWide, 8>(p, warps, sms, s);
  if constexpr (!kWide) {
    if (each <= 16) return forward_items<T, W, false, 16>(p, warps, sms, s);
    forward_items<T, W, false, 32>(p, warps, sms, s);
  }
}

template <typename T, typename W>
void launch_forward(const NormParams& p, int dev, int sms, cudaStream_t s) {
  if (wide_rows(p.x, p.ld, p.H, sizeof(T)) && wide_rows(p.out, p.ld_out, p.H, sizeof(T)))
    forward<T, W, true>(p, dev, sms, s);
  else
    forward<T, W, false>(p, dev, sms, s);
}

template <typename T, typename W, bool kWide, int kElems>
bool grad(const NormParams& p, const NormPlan& plan, cudaStream_t s) {
  const int units = plan.threads == 32 ? 8 : 1;  // of a CTA
  const int grid = (plan.parts + units - 1) / units, threads = plan.threads * units;
  norm_grad_kernel<T, W, kWide, kElems><<<grid, threads, 0, s>>>(p, plan.threads);
  return cudaGetLastError() == cudaSuccess;
}

// Rows that lie alike, one for every SM and more: a CTA to an SM, as many units
// in it as there are rows and threads for.  False: no such rows, or no room for two: the
// ring's places are 512 threads apart whatever the unit, so float32 above 8192 columns has none.
template <typename T, typename W, int kElems, bool kEdges>
bool grad_ring(const NormParams& p, int dev, cudaStream_t s) {
  constexpr int kMore = kEdges ? 16 / sizeof(T) - 1 : 0;  // columns in front of a row
  const int span = (p.H + kMore + kElems * 32 - 1) / (kElems * 32) * 32, rows = (p.M + kNormSms - 1) / kNormSms;
  const int units = std::min(kNormRingThreads / span, rows);
  const int threads = units * span, row = kNormRingThreads * kElems * 2 * static_cast<int>(sizeof(T));
  const int staged = kElems <= 16 ? 0 : staged_cols(p.H + kMore) * static_cast<int>(sizeof(float));
  const int ring = units ? std::min(8, (kMostShared - staged) / row) : 0;
  // (it leaves a part of every SM's: no fewer may have room)
  if (ring < 2 || p.parts < kNormSms || !open_shared<norm_grad_ring_kernel<T, W, kElems, kEdges>>(dev, kMostShared)) return false;
  const int smem = std::max(ring * row + staged, units * 2 * p.H * static_cast<int>(sizeof(float)));
  norm_grad_ring_kernel<T, W, kElems, kEdges><<<kNormSms, threads, smem, s>>>(p, span, ring);
  return true;
}

// 16384 rows of 4096 bf16, eight elements to a thread: 100 us, sixteen: 76; float32: 127
// and 140.  100000 rows of 128 bf16: 31 and 39.  16384 of 4608 bf16, sixteen: 118, thirty-two,
// which leave room for more units: 95; 8192 of 4608 float32: 79 and 117.
template <typename T, typename W, bool kEdges>
bool grad_rings(const NormParams& p, int dev, cudaStream_t s) {
  const bool bf16 = sizeof(T) == 2;
  const int H = p.H + (kEdges ? 16 / sizeof(T) - 1 : 0);
  return H <= (bf16 ? 256 : 4096)    ? grad_ring<T, W, 8, kEdges>(p, dev, s)
         : H <= (bf16 ? 4096 : 8192) ? grad_ring<T, W, 16, kEdges>(p, dev, s)
                                     : grad_ring<T, W, 32, kEdges>(p, dev, s);
}

// Sets the number of parts that it leaves.
template <typename T, typename W, bool kWide>
bool backward(NormParams& p, int dev, cudaStream_t s) {
  // Rows that start anywhere, an element at a time otherwise: 1000 of 4099 bf16 25 us (64); few
  // of float32 not: 2000 of 1027 17 us (14), 4000 20 (21); measured at that width alone.
  const bool edges = !kWide && p.H >= 64 && (sizeof(T) == 2 || p.M >= 32 * kNormSms) && alike(p.x, p.ld, p.gy, p.ld_gy, sizeof(T)) &&
                     (!p.out || alike(p.x, p.ld, p.out, p.ld_out, sizeof(T)));
  if ((kWide || edges) && grad_rings<T, W, !kWide>(p, dev, s)) {
    p.parts = kNormSms;  // of p.parts, which is parts_of(M, H) and the workspace's: as many or more
    return cudaGetLastError() == cudaSuccess;
  }
  const NormPlan plan = norm_plan(p.M, p.H);
  return plan.elems == 8    ? grad<T, W, kWide, 8>(p, plan, s)
         : plan.elems == 16 ? grad<T, W, kWide, 16>(p, plan, s)
                            : grad<T, W, kWide, 32>(p, plan, s);
}

template <typename T, typename W>
int launch_backward(NormParams p, int dev, cudaStream_t s) {
  if (p.M) {
    const bool wide = wide_rows(p.x, p.ld, p.H, sizeof(T)) && wide_rows(p.gy, p.ld_gy, p.H, sizeof(T)) &&
                      (!p.out || wide_rows(p.out, p.ld_out, p.H, sizeof(T)));
    if (!(wide ? backward<T, W, true>(p, dev, s) : backward<T, W, false>(p, dev, s))) return CAI_ERR_CUDA;
  }
  if (!p.gw && !p.gb) return CAI_OK;
  // The sums' kernel is launched while the other runs, and waits for its end.
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((p.H + 31) / 32);
  cfg.blockDim = dim3(32 * kNormSumWarps);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = p.M ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, norm_weight_sum_kernel<W>, p) != cudaSuccess) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  return CAI_OK;
}

}  // namespace

extern "C" int cai_norm_rows(const void* x, int32_t dtype, int64_t ld, int32_t M, int32_t H,
                             int32_t kind, const void* weight, const void* bias, int32_t wdtype,
                             double eps, void* y, int64_t ld_y, float* stats, void* stream) {
  int r = check_norm(x, dtype, ld, M, H, kind, wdtype);
  if (r != CAI_OK) return r;
  const float e32 = static_cast<float>(eps);
  if (!(e32 > 0.0f) || !std::isfinite(e32)) return CAI_ERR_ARG;
  if (M == 0) return CAI_OK;
  const int e = elem_bytes(dtype), we = elem_bytes(wdtype);
  if (!y || ld_y < H || !aligned_to(y, e) || !may_write(y, ld_y, x, ld, e, M, H)) return CAI_ERR_ARG;
  const uint64_t y_bytes = rows_bytes(ld_y, M, H, e), s_bytes = 8ull * M, w_bytes = static_cast<uint64_t>(H) * we;
  if (bytes_overlap(stats, s_bytes, x, rows_bytes(ld, M, H, e)) || bytes_overlap(stats, s_bytes, y, y_bytes))
    return CAI_ERR_ARG;
  int dev = 0, sms = 0;
  if ((r = this_device(&dev, &sms)) != CAI_OK) return r;
  if (!on_this_device(x, dev) || !on_this_device(y, dev)) return CAI_ERR_ARG;
  const void* ptrs[] = {weight, bias, stats};
  for (const void* q : ptrs)
    if (q && (!aligned_to(q, q == stats ? 4 : we) || !on_this_device(q, dev) ||
              (q != stats && (bytes_overlap(q, w_bytes, y, y_bytes) || bytes_overlap(q, w_bytes, stats, s_bytes)))))
      return CAI_ERR_ARG;
  NormParams p = {};
  p.x = x;
  p.ld = ld;
  p.M = M;
  p.H = H;
  p.layer = kind == CAI_NORM_LAYER;
  p.weight = weight;
  p.bias = bias;
  p.eps = e32;
  p.stats = stats;
  p.out = y;
  p.ld_out = ld_y;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  using bf16 = __nv_bfloat16;
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (dtype == CAI_BF16)
    wdtype == CAI_BF16 ? launch_forward<bf16, bf16>(p, dev, sms, s) : launch_forward<bf16, float>(p, dev, sms, s);
  else
    wdtype == CAI_BF16 ? launch_forward<float, bf16>(p, dev, sms, s) : launch_forward<float, float>(p, dev, sms, s);
  return launched();
}

extern "C" int cai_norm_workspace(int32_t M, int32_t H, int64_t* bytes) {
  if (!bytes) return CAI_ERR_ARG;
  if (M < 0 || H < 1 || H > kNormMaxH) return CAI_ERR_SHAPE;
  *bytes = static_cast<int64_t>(parts_of(M, H)) * 2 * H * sizeof(float);
  return CAI_OK;
}

extern "C" int cai_norm_backward(const void* x, int32_t dtype, int64_t ld, const void* grad_y,
                                 int64_t ld_gy, int32_t M, int32_t H, int32_t kind,
                                 const void* weight, int32_t wdtype, const float* stats,
                                 void* grad_x, int64_t ld_gx, void* grad_weight, void* grad_bias,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
  int r = check_norm(x, dtype, ld, M, H, kind, wdtype);
  if (r != CAI_OK) return r;
  const int e = elem_bytes(dtype), we = elem_bytes(wdtype);
  const bool sums = grad_weight || grad_bias;
  if (!grad_x && !sums && M != 0) return CAI_ERR_ARG;
  if (!grad_x && !sums) return CAI_OK;
  if (M != 0) {
    if (!grad_y || !stats || ld_gy < H || !aligned_to(grad_y, e)) return CAI_ERR_ARG;
    if (grad_x && (ld_gx < H || !aligned_to(grad_x, e) || !may_write(grad_x, ld_gx, x, ld, e, M, H) ||
                   !may_write(grad_x, ld_gx, grad_y, ld_gy, e, M, H)))
      return CAI_ERR_ARG;
  }
  int64_t need = 0;
  cai_norm_workspace(M, H, &need);
  if (sums && need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16))) return CAI_ERR_ARG;
  // What is written, against everything else.
  const Part part[] = {
      {workspace, sums ? static_cast<uint64_t>(need) : 0, true},
      {grad_weight, static_cast<uint64_t>(H) * we, true},
      {grad_bias, static_cast<uint64_t>(H) * we, true},
      {M ? grad_x : nullptr, M ? rows_bytes(ld_gx, M, H, e) : 0, true},
      {M ? x : nullptr, M ? rows_bytes(ld, M, H, e) : 0, false},
      {M ? grad_y : nullptr, M ? rows_bytes(ld_gy, M, H, e) : 0, false},
      {weight, static_cast<uint64_t>(H) * we, false},
      {M ? stats : nullptr, 8ull * M, false},
  };
  if (parts_overlap(part, 8, 3, 4, 5)) return CAI_ERR_ARG;  // (rows against rows have been looked at)
  int dev = 0, sms = 0;
  if ((r = this_device(&dev, &sms)) != CAI_OK) return r;
  for (const Part& q : part)
    if (q.p && q.bytes && !on_this_device(q.p, dev)) return CAI_ERR_ARG;
  if (!aligned_to(grad_weight, we) || !aligned_to(grad_bias, we) || !aligned_to(weight, we) || !aligned4(stats))
    return CAI_ERR_ARG;
  NormParams p = {};
  p.x = x;
  p.ld = ld;
  p.gy = grad_y;
  p.ld_gy = ld_gy;
  p.M = M;
  p.H = H;
  p.layer = kind == CAI_NORM_LAYER;
  p.weight = weight;
  p.stats = const_cast<float*>(stats);
  p.out = grad_x;
  p.ld_out = ld_gx;
  p.part = sums ? static_cast<float*>(workspace) : nullptr;
  p.parts = parts_of(M, H);
  p.gw = grad_weight;
  p.gb = grad_bias;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  using bf16 = __nv_bfloat16;
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (dtype == CAI_BF16)
    return wdtype == CAI_BF16 ? launch_backward<bf16, bf16>(p, dev, s) : launch_backward<bf16, float>(p, dev, s);
  return wdtype == CAI_BF16 ? launch_backward<float, bf16>(p, dev, s) : launch_backward<float, float>(p, dev, s);
}
