// Host side of the losses on drawn tokens declared in include/cai.h: argument
// checks and launches.  They keep no state and need no workspace.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "cai.h"
#include "host_checks.h"
#include "policy.cuh"

using namespace cai;

namespace {

// Each kernel is launched while the one before it in the stream ends, and waits for its
// end before it reads or writes anything.
void after_previous(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at) {
  at[cfg->numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[cfg->numAttrs].val.programmaticStreamSerializationAllowed = 1;
  cfg->attrs = at;
  ++cfg->numAttrs;
}

template <typename... A>
int launch(void (*kernel)(A...), unsigned grid, unsigned threads, void* stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[1];
  after_previous(&cfg, at);
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  return CAI_OK;
}

// What the rows kernels may take of each device, found on first use.
struct TokenDevice {
  bool ready = false;
  int sms = 0;
  int limit = 0;                  // dynamic shared memory of a CTA
  int clusters[2][2][4][6] = {};  // resident at once: by type, gradient, log2 of a cluster's CTAs, shape
};
std::mutex g_token_mutex;
TokenDevice g_token[kMaxDevices];

// Threads of a CTA and CTAs of an SM that the rows kernels come in.  2048 rows of 126464
// bf16, all with a part, the best cut of each, in an earlier form that took 188 us where this one
// takes 169: loss and gradient 187 us (128 x 3), 188 (x 5), 191 (x 4), 197 (256 x 2 and 512 x 1),
// of 152 at the copy's rate; 64 registers instead of 128, so that more warps fit, 202
// to 218.  The losses alone 86 (256 x 4), 85 (128 x 8), 90 (512 x 2), of 76.  Fewer threads
// are for short rows: 20000 of 4096 bf16, the losses 129 us (128 x 8) and 41 (64 x 12).
struct Shape {
  int threads, share;
};
constexpr int kMostShapes = 6;
constexpr Shape kShapes[2][kMostShapes] = {{{256, 4}, {128, 8}, {64, 12}, {32, 16}},
                                           {{128, 2}, {128, 3}, {128, 4}, {128, 5}, {64, 8}, {32, 16}}};
constexpr int kShapeCount[2] = {4, 6};

size_t ring_bytes(int ring, int threads) { return static_cast<size_t>(ring) * kBatch * threads * 16; }
// Batches that a CTA's part of an SM's shared memory has room for.
int most_ring(int limit, const Shape& s) {
  constexpr int kStatic = sizeof(TokenShared) + 1024;  // a CTA's shared memory beside the ring: its own, the system's
  return ((limit + kStatic) / s.share - kStatic) / static_cast<int>(ring_bytes(1, s.threads));
}

void cluster_of(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int ctas) {
  at->id = cudaLaunchAttributeClusterDimension;
  at->val.clusterDim.x = ctas;
  at->val.clusterDim.y = 1;
  at->val.clusterDim.z = 1;
  cfg->attrs = at;
  cfg->numAttrs = ctas > 1 ? 1 : 0;
}

template <typename T, bool kGrad, TokenEnds kEnds>
bool open_rows(int optin, TokenDevice* d) {
  auto* kernel = token_rows_kernel<T, kGrad, kEnds>;
  cudaFuncAttributes a{};
  if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess) return false;
  const int n = optin - static_cast<int>(a.sharedSizeBytes);
  if (d->limit == 0 || n < d->limit) d->limit = n;
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, n) == cudaSuccess &&
         cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) ==
             cudaSuccess;
}

template <typename T>
bool open_all(int optin, TokenDevice* d) {
  return open_rows<T, true, kWhole>(optin, d) && open_rows<T, true, kCut>(optin, d) &&
         open_rows<T, true, kShifted>(optin, d) && open_rows<T, false, kWhole>(optin, d) && open_rows<T, false, kCut>(optin, d);
}

// Clusters that are resident at once, for every size of them.
template <typename T, bool kGrad>
void count_clusters(int sms, TokenDevice* d) {
  for (int c = 0; c < 4; ++c)
    for (int k = 0; k < kShapeCount[kGrad]; ++k) {
      const Shape& s = kShapes[kGrad][k];
      const int most = sms * s.share >> c;
      int& known = d->clusters[sizeof(T) == 2][kGrad][c][k];
      known = most > 0 ? most : 1;
      const size_t smem = ring_bytes(most_ring(d->limit, s), s.threads);
      int n = 0;
      if (c == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, token_rows_kernel<T, kGrad, kCut>, s.threads, smem) ==
                cudaSuccess && n > 0 && n < s.share)
          known = n * sms;
        cudaGetLastError();
        continue;
      }
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute at[1];
      cfg.gridDim = dim3(static_cast<unsigned>(known << c));
      cfg.blockDim = dim3(s.threads);
      cfg.dynamicSmemBytes = smem;
      cluster_of(&cfg, at, 1 << c);
      if (cudaOccupancyMaxActiveClusters(&n, token_rows_kernel<T, kGrad, kCut>, &cfg) == cudaSuccess && n > 0 && n < known)
        known = n;
      cudaGetLastError();
    }
}

int token_device(int* dev, TokenDevice** out) {
  int sms = 0;
  const int r = this_device(dev, &sms);
  if (r != CAI_OK) return r;
  TokenDevice& d = g_token[*dev];
  std::lock_guard<std::mutex> lock(g_token_mutex);
  if (!d.ready) {
    int optin = 0;
    d.sms = sms;
    if (cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, *dev) != cudaSuccess ||
        !open_all<float>(optin, &d) || !open_all<__nv_bfloat16>(optin, &d)) {
      cudaGetLastError();
      return CAI_ERR_CUDA;
    }
    count_clusters<float, true>(sms, &d);
    count_clusters<float, false>(sms, &d);
    count_clusters<__nv_bfloat16, true>(sms, &d);
    count_clusters<__nv_bfloat16, false>(sms, &d);
    d.ready = true;
  }
  *out = &d;
  return CAI_OK;
}

// How a row is cut, and by which shape of CTAs: the cut of the least time by a model of
// it.  A round of the clusters takes the rows' bytes at the SM's share of the memory's
// rate, or what one CTA's work takes from a row to the next where that is more: its
// reduction (and the other CTAs' sums), and its batches one after another.  With the
// gradient a slice stays in the ring, and some of another comes meanwhile; no plan
// (threads 0) where none has room.
template <typename T, bool kGrad>
TokenPlan token_plan(int M, int V, bool aligned, const TokenDevice& d) {
  constexpr double kRate = 42.0, kRow = 1.2, kTold = 2.5, kLatency = 2.4;  // bytes a ns, us
  TokenPlan best = {};
  double least = 1e30;
  for (int k = 0; k < kShapeCount[kGrad]; ++k) {
    const Shape& s = kShapes[kGrad][k];
    const int batch = s.threads * kBatch;
    for (int ic = 0; 1 << ic <= kRowMaxCluster; ++ic) {
      const int c = 1 << ic;
      if (c > 1 && V / c < 1024) break;
      const int n = row_chunk(V, c) / Row<T>::kVec + (aligned ? 0 : 2);
      TokenPlan plan = {c, s.threads, (n + batch - 1) / batch, most_ring(d.limit, s), 0, -1};
      if (plan.ring > 3 * plan.batches - 1) plan.ring = 3 * plan.batches - 1;
      if (plan.ring > (kGrad ? plan.batches : 0) + 7) plan.ring = (kGrad ? plan.batches : 0) + 7;
      if (kGrad && plan.ring <= plan.batches) continue;
      const int clusters = d.clusters[sizeof(T) == 2][kGrad][ic][k];
      const int rounds = (M + clusters - 1) / clusters;
      // (rounds after the first find their logits there)
      const int busy = static_cast<int>((static_cast<long long>(M < clusters ? M : clusters) * c + d.sms - 1) / d.sms);
      const double bytes = n * 16.0 * (kGrad ? 2 : 1) * busy / kRate * 1e-3;
      const double batch_time = kGrad ? 0.9 : std::max(0.4, kLatency / plan.ring);
      const double work = kRow + (c > 1 ? kTold : 0.0) + plan.batches * batch_time;
      const double time = rounds * (bytes > work ? bytes : work);
      if (time < least) {
        least = time;
        best = plan;
        best.clusters = M < clusters ? M : clusters;
      }
    }
  }
  return best;
}

template <typename T, bool kGrad, TokenEnds kEnds, bool kLate = false>
int launch_rows(const TokenParams& p, const TokenPlan& plan, void* stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(plan.clusters * plan.ctas));
  cfg.blockDim = dim3(plan.threads);
  cfg.dynamicSmemBytes = ring_bytes(plan.ring, plan.threads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[2];
  cluster_of(&cfg, at, plan.ctas);
  after_previous(&cfg, at);
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (cudaLaunchKernelEx(&cfg, token_rows_kernel<T, kGrad, kEnds, kLate>, p, plan) != cudaSuccess) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  return CAI_OK;
}

template <typename T>
int launch_grad(const TokenParams& p, void* stream) {
  const int most = 1024 * Row<T>::kVec;  // elements of a CTA
  const int parts = (p.V + most - 1) / most;
  const int chunk = row_chunk(p.V, parts);
  return launch(token_grad_kernel<T>, static_cast<unsigned>(p.M) * parts, 256, stream, p, parts, chunk);
}

// Losses and, where it is asked for, the gradient: in one kernel where a row fits the
// shared memory.
template <typename T>
int run_rows(const TokenParams& p, const TokenDevice& d, void* stream) {
  const bool alike = (reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.grad)) % 16 == 0 &&
                     (p.M == 1 || (p.ld - p.ld_grad) * static_cast<int64_t>(sizeof(T)) % 16 == 0);
  const bool aligned = aligned_to(p.logits, 16) && (p.M == 1 || p.ld * static_cast<int64_t>(sizeof(T)) % 16 == 0);
  const bool whole = aligned && p.V * sizeof(T) % 16 == 0;  // rows of whole vectors
  if (p.grad) {
    const TokenPlan plan = token_plan<T, true>(p.M, p.V, aligned, d);
    // bf16 that has to be moved along, with a fifth of a cut's places empty: two kernels, 300
    // rows of 50003, a quarter empty, 22 us (25), 600 43 (45); 300 of 126465, a thirtieth
    // empty, 51 (47).  (The border between is not measured.)
    const int vectors = plan.threads ? row_chunk(p.V, plan.ctas) / Row<T>::kVec : 0;
    const bool loose = !alike && sizeof(T) == 2 && plan.clusters < p.M &&
                       5 * vectors < 4 * plan.batches * kBatch * plan.threads;
    if (plan.threads && !loose)
      return !alike  ? launch_rows<T, true, kShifted>(p, plan, stream)
             : whole ? launch_rows<T, true, kWhole>(p, plan, stream)
                     : launch_rows<T, true, kCut>(p, plan, stream);
  }
  const TokenPlan plan = token_plan<T, false>(p.M, p.V, aligned, d);
  const int r = whole ? launch_rows<T, false, kWhole>(p, plan, stream) : launch_rows<T, false, kCut>(p, plan, stream);
  return r == CAI_OK && p.grad ? launch_grad<T>(p, stream) : r;
}

// Everything but what a loss needs beside its rows; 1: no rows, done.
int check(const TokenParams& p, int32_t dtype, TokenDevice** d) {
  // (a row of V has up to 64 parts in the gradient kernel's grid)
  int r = check_rows(p.logits, dtype, p.ld, p.M, p.V, 64);
  if (r != CAI_OK) return r;
  if (!is_temperature(p.tau)) return CAI_ERR_ARG;
  if (p.M == 0) return 1;
  const int e = elem_bytes(dtype);
  if (p.grad) {
    if (p.ld_grad < p.V || !aligned_to(p.grad, e)) return CAI_ERR_ARG;
    if ((p.grad != p.logits || p.ld_grad != p.ld) &&
        rows_overlap(p.logits, p.ld, e, p.grad, p.ld_grad, e, p.M, p.V))
      return CAI_ERR_ARG;
  }
  // (rows against rows have been looked at; stats and slope are the loss's to write)
  const uint64_t n = 4ull * p.M;
  const bool loss = p.logp != nullptr;
  const Part part[] = {{p.grad, p.grad ? rows_bytes(p.ld_grad, p.M, p.V, e) : 0, true},
                       {p.logits, rows_bytes(p.ld, p.M, p.V, e), false},
                       {p.token, n, false},
                       {p.old_logp, n, false},
                       {p.advantage, n, false},
                       {p.ref_logp, n, false},
                       {p.weight, n, false},
                       {p.upstream, n, false},
                       {p.loss, n, true},
                       {p.logp, n, true},
                       {p.stats, 2 * n, loss},
                       {p.slope, n, loss}};
  if (parts_overlap(part, 12, 0, 1, 1)) return CAI_ERR_ARG;
  int dev = 0;
  if ((r = token_device(&dev, d)) != CAI_OK) return r;
  const void* ptrs[] = {p.token, p.old_logp, p.advantage, p.ref_logp, p.weight,
                        p.loss,  p.logp,     p.stats,     p.slope,    p.upstream};
  for (const void* q : ptrs)
    if (q && (!aligned4(q) || !on_this_device(q, dev))) return CAI_ERR_ARG;
  if (!on_this_device(p.logits, dev) || (p.grad && !on_this_device(p.grad, dev))) return CAI_ERR_ARG;
  return CAI_OK;
}

TokenParams rows_of(const void* logits, int64_t ld, int32_t M, int32_t V, const int32_t* token,
                    double temperature) {
  TokenParams p = {};
  p.logits = logits;
  p.ld = ld;
  p.M = M;
  p.V = V;
  p.token = token;
  p.tau = static_cast<float>(temperature);
  p.inv_tau = 1.0 / p.tau;
  return p;
}

int backward(TokenParams& p, int32_t dtype, void* stream) {
  TokenDevice* d = nullptr;
  const int r = check(p, dtype, &d);
  if (r != CAI_OK) return r == 1 ? CAI_OK : r;
  if (!p.token || !p.stats || !p.upstream || !p.grad) return CAI_ERR_ARG;
  return dtype == CAI_BF16 ? launch_grad<__nv_bfloat16>(p, stream) : launch_grad<float>(p, stream);
}

}  // namespace

extern "C" int cai_token_logp(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                              const int32_t* token, double temperature, float* logp, float* stats,
                              void* stream) {
  TokenParams p = rows_of(logits, ld, M, V, token, temperature);
  p.logp = logp;
  p.stats = stats;
  TokenDevice* d = nullptr;
  const int r = check(p, dtype, &d);
  if (r != CAI_OK) return r == 1 ? CAI_OK : r;
  if (!token || !logp || !stats) return CAI_ERR_ARG;
  return dtype == CAI_BF16 ? run_rows<__nv_bfloat16>(p, *d, stream) : run_rows<float>(p, *d, stream);
}

extern "C" int cai_token_logp_backward(const void* logits, int32_t dtype, int64_t ld, int32_t M,
                                       int32_t V, const int32_t* token, double temperature,
                                       const float* stats, const float* grad_logp, void* grad,
                                       int64_t ld_grad, void* stream) {
  TokenParams p = rows_of(logits, ld, M, V, token, temperature);
  p.stats = const_cast<float*>(stats);
  p.upstream = grad_logp;
  p.grad = grad;
  p.ld_grad = ld_grad;
  return backward(p, dtype, stream);
}

extern "C" int cai_policy_loss(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                               const int32_t* token, const float* old_logp, const float* advantage,
                               const float* ref_logp, const float* weight, double temperature,
                               double clip_low, double clip_high, double kl, float* loss, float* logp,
                               float* stats, float* slope, void* grad, int64_t ld_grad,
                               void* stream) {
  TokenParams p = rows_of(logits, ld, M, V, token, temperature);
  p.policy = true;
  p.old_logp = old_logp;
  p.advantage = advantage;
  p.ref_logp = ref_logp;
  p.weight = weight;
  p.low = static_cast<float>(1.0 - clip_low);
  p.high = static_cast<float>(1.0 + clip_high);
  p.kl = static_cast<float>(kl);
  p.loss = loss;
  p.logp = logp;
  p.stats = stats;
  p.slope = slope;
  p.grad = grad;
  p.ld_grad = ld_grad;
  if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(p.high) ||
      !std::isfinite(p.kl))
    return CAI_ERR_ARG;
  TokenDevice* d = nullptr;
  int r = check(p, dtype, &d);
  if (r != CAI_OK) return r == 1 ? CAI_OK : r;
  if (!token || !advantage || !loss || !logp || !stats || !slope || (p.kl != 0.0f && !ref_logp))
    return CAI_ERR_ARG;
  return dtype == CAI_BF16 ? run_rows<__nv_bfloat16>(p, *d, stream) : run_rows<float>(p, *d, stream);
}

extern "C" int cai_policy_backward(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V,
                                   const int32_t* token, double temperature, const float* stats,
                                   const float* slope, const float* grad_loss, void* grad,
                                   int64_t ld_grad, void* stream) {
  TokenParams p = rows_of(logits, ld, M, V, token, temperature);
  p.stats = const_cast<float*>(stats);
  p.slope = const_cast<float*>(slope);
  p.upstream = grad_loss;
  p.grad = grad;
  p.ld_grad = ld_grad;
  if (M != 0 && !slope) return CAI_ERR_ARG;
  return backward(p, dtype, stream);
}

extern "C" int cai_test_late_rows(const float* logits, int32_t M, int32_t V, const int32_t* token,
                                  const float* advantage, int32_t ctas, int32_t late_row, float* loss,
                                  float* logp, float* stats, float* slope, float* grad, void* stream) {
  TokenParams p = rows_of(logits, V, M, V, token, 1.0);
  p.policy = true;
  p.advantage = advantage;
  p.low = p.high = 1.0f;
  p.loss = loss;
  p.logp = logp;
  p.stats = stats;
  p.slope = slope;
  p.grad = grad;
  p.ld_grad = V;
  if (ctas < 2 || ctas > kRowMaxCluster || (ctas & (ctas - 1)) || V < 1024 * ctas || V > 4096 * ctas || V % 4 || M < 1 ||
      late_row < 0 || late_row >= M)
    return CAI_ERR_SHAPE;
  if (!aligned_to(logits, 16) || !aligned_to(grad, 16)) return CAI_ERR_ARG;
  TokenDevice* d = nullptr;
  const int r = check(p, CAI_F32, &d);
  if (r != CAI_OK) return r;
  if (!token || !advantage || !loss || !logp || !stats || !slope) return CAI_ERR_ARG;
  // One cluster, so that rows are taken one after another.
  constexpr int kThreads = 128;
  TokenPlan plan = {ctas, kThreads, 0, 0, 1, late_row};
  plan.batches = (row_chunk(V, ctas) / 4 + kThreads * kBatch - 1) / (kThreads * kBatch);
  plan.ring = plan.batches + 1;
  return grad ? launch_rows<float, true, kWhole, true>(p, plan, stream)
              : launch_rows<float, false, kWhole, true>(p, plan, stream);
}

extern "C" int cai_preference_loss(const float* logp, const float* ref_logp, const float* weight,
                                   const int32_t* offsets, int32_t M, int32_t pairs, double beta,
                                   double smoothing, const float* grad_loss, float* loss,
                                   float* margin, float* grad_logp, void* stream) {
  PairParams p{logp, ref_logp, weight, offsets, M, pairs, static_cast<float>(beta),
               static_cast<float>(smoothing), grad_loss, loss, margin, grad_logp};
  if (!std::isfinite(p.beta) || !(smoothing >= 0.0 && smoothing <= 1.0)) return CAI_ERR_ARG;
  if (M < 0 || pairs < 0 || pairs > (1 << 30)) return CAI_ERR_SHAPE;
  if (!offsets || (M != 0 && !logp) || (pairs != 0 && (!loss || !margin))) return CAI_ERR_ARG;
  const uint64_t n = 4ull * M, k = 4ull * pairs;
  const Part part[] = {{grad_logp, n, true}, {loss, k, true}, {margin, k, true}, {grad_loss, k, false},
                       {logp, n, false}, {ref_logp, n, false}, {weight, n, false}, {offsets, 2 * k + 4, false}};
  if (parts_overlap(part, 8, -1, -1, -1)) return CAI_ERR_ARG;
  int dev = 0, sms = 0;
  const int r = this_device(&dev, &sms);
  if (r != CAI_OK) return r;
  const void* ptrs[] = {logp, ref_logp, weight, offsets, grad_loss, loss, margin, grad_logp};
  for (const void* q : ptrs)
    if (q && (!aligned4(q) || !on_this_device(q, dev))) return CAI_ERR_ARG;
  return launch(preference_kernel, static_cast<unsigned>(pairs) + 1, kPairThreads, stream, p);
}
