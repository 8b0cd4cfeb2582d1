// Host side of the 4-bit LM head declared in include/cai.h (cai_mx4_*): the
// handle with the packed weight and the workspace of the packed rows, argument
// checks and launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <new>

#include "cai.h"
#include "internal.h"
#include "mx4.cuh"

using namespace cai;

struct cai_mx4 {
  int dev = 0, sms = 0;
  int V = 0, H = 0, KB = 0, max_rows = 0;
  int tile = 0, n_vt = 0;
  size_t smem_limit = 0;       // dynamic shared memory a launch may ask for
  uint8_t* w = nullptr;        // packed weight
  uint8_t* rows = nullptr;     // packed rows of the call in progress
  int pairs = 0;               // CTA pairs resident at once
  int pair_stages[2] = {};     // by the logits' size: 2 bytes, 4
  Mx4PairMaps maps;
  uint32_t* err = nullptr;     // mapped host memory: bits of waits that gave up
  uint32_t* d_err = nullptr;   // its device address
};

namespace {

bool on_device(const void* p, int dev) {
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return (a.type == cudaMemoryTypeDevice || a.type == cudaMemoryTypeManaged) && a.device == dev;
}

int elem_bytes(int dtype) { return dtype == CAI_BF16 ? 2 : dtype == CAI_F32 ? 4 : 0; }

// The device of the handle has to be the current one, and no wait given up.
int usable(const cai_mx4* h) {
  if (!h) return CAI_ERR_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  if (dev != h->dev) return CAI_ERR_ARG;
  return *reinterpret_cast<volatile uint32_t*>(h->err) ? CAI_ERR_DEVICE : CAI_OK;
}

// Vocabulary rows per tile: as few turns over the SMs as tiles of kMx4MaxTile rows
// allow, and then tiles as narrow as that many turns allow, so that every SM
// gets the same share of W.
int tile_rows(int V, int sms) {
  const int turns = (V + sms * kMx4MaxTile - 1) / (sms * kMx4MaxTile);
  const int n = (V + sms * turns - 1) / (sms * turns);
  const int t = (n + 15) / 16 * 16;
  return t < 16 ? 16 : t;
}

int pack(const cai_mx4* h, const void* src, int dtype, long long rows, long long rows_pad, int tile,
         uint8_t* dst, void* values, cudaStream_t stream) {
  Mx4PackParams p{src, dst, static_cast<__nv_bfloat16*>(values), rows, rows_pad, h->H, h->KB, tile};
  const long long blocks = (rows_pad * 2 * h->KB + 31) / 32;
  const int grid = static_cast<int>(blocks < h->sms * 256ll ? blocks : h->sms * 256ll);
  cudaGetLastError();  // an error left by earlier work is not this call's
  if (dtype == CAI_BF16)
    mx4_pack_kernel<__nv_bfloat16><<<grid, 256, 0, stream>>>(p);
  else
    mx4_pack_kernel<float><<<grid, 256, 0, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return CAI_ERR_CUDA;
  return CAI_OK;
}

template <typename T>
bool launch_product(const Mx4Params& p, int grid, size_t smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kMx4Threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, mx4_logits_kernel<T>, p) == cudaSuccess;
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                             const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Packed bytes as rows of 128, copied `box` rows at a time as they lie.
bool encode_rows(EncodeFn fn, CUtensorMap* m, void* base, size_t bytes, int box) {
  cuuint64_t dims[2] = {128, bytes / 128};
  cuuint64_t strides[1] = {128};
  cuuint32_t boxes[2] = {128, static_cast<cuuint32_t>(box)};
  cuuint32_t ones[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, boxes, ones,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The pair kernel's maps, stages and resident pairs.
int set_up_pairs(cai_mx4* h, size_t w_bytes, size_t r_bytes) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
          cudaSuccess ||
      q != cudaDriverEntryPointSuccess)
    return CAI_ERR_CUDA;
  const EncodeFn encode = reinterpret_cast<EncodeFn>(fn);
  if (!encode_rows(encode, &h->maps.rows, h->rows, r_bytes, mx4_stage_bytes(kMx4RowTile) / 128) ||
      !encode_rows(encode, &h->maps.w, h->w, w_bytes, h->tile / 2) ||
      !encode_rows(encode, &h->maps.scales, h->w, w_bytes, mx4_scale_bytes(h->tile) / 128))
    return CAI_ERR_CUDA;
  for (int k = 0; k < 2; ++k) {
    int n = kMx4MaxStages;
    while (n > 2 && mx4_pair_smem_bytes(n, h->tile, 2 << k) > h->smem_limit) --n;
    h->pair_stages[k] = n;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(h->sms & ~1));
  cfg.blockDim = dim3(kMx4Threads);
  cfg.dynamicSmemBytes = mx4_pair_smem_bytes(h->pair_stages[1], h->tile, 4);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&h->pairs, mx4_logits_pair_kernel<float>, &cfg) != cudaSuccess ||
      h->pairs < 1)
    return CAI_ERR_CUDA;
  return CAI_OK;
}

template <typename T>
bool launch_pairs(const cai_mx4* h, const Mx4Params& p, int grid, size_t smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kMx4Threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 2;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, mx4_logits_pair_kernel<T>, h->maps, p) == cudaSuccess;
}

template <typename K>
bool open_smem(K* kernel, int optin, size_t* limit) {
  cudaFuncAttributes a{};
  if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess) return false;
  const size_t n = static_cast<size_t>(optin) - a.sharedSizeBytes;
  if (*limit == 0 || n < *limit) *limit = n;
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(n)) == cudaSuccess;
}

int check_weight(const cai_mx4* h, const void* W, int32_t dtype, const void* values) {
  if (!W || !elem_bytes(dtype)) return CAI_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(W) % 16 != 0 || reinterpret_cast<uintptr_t>(values) % 16 != 0)
    return CAI_ERR_ARG;
  if (!on_device(W, h->dev) || (values && !on_device(values, h->dev))) return CAI_ERR_ARG;
  return CAI_OK;
}

int init(cai_mx4* h, const void* W, int32_t dtype, cudaStream_t stream) {
  int major = 0, minor = 0, optin = 0;
  if (cudaGetDevice(&h->dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, h->dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, h->dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, h->dev) != cudaSuccess)
    return CAI_ERR_CUDA;
  if (major != 10 || minor != 3) return CAI_ERR_UNSUPPORTED;
  int r = check_weight(h, W, dtype, nullptr);
  if (r != CAI_OK) return r;
  if (!open_smem(mx4_logits_pair_kernel<float>, optin, &h->smem_limit) ||
      !open_smem(mx4_logits_pair_kernel<__nv_bfloat16>, optin, &h->smem_limit) ||
      !open_smem(mx4_logits_kernel<float>, optin, &h->smem_limit) ||
      !open_smem(mx4_logits_kernel<__nv_bfloat16>, optin, &h->smem_limit))
    return CAI_ERR_CUDA;
  h->KB = (h->H + kMx4K - 1) / kMx4K;
  h->tile = tile_rows(h->V, h->sms);
  h->n_vt = (h->V + h->tile - 1) / h->tile;
  const size_t w_bytes = static_cast<size_t>(h->n_vt) * h->KB * mx4_stage_bytes(h->tile);
  size_t n_mt = (h->max_rows + kMx4RowTile - 1) / kMx4RowTile;
  if (n_mt > 1) n_mt = (n_mt + 1) / 2 * 2;  // whole tiles of the pair kernel
  const size_t r_bytes = n_mt * h->KB * mx4_stage_bytes(kMx4RowTile);
  void* p = nullptr;
  if ((r = device_alloc(&p, w_bytes)) != CAI_OK) return r;
  h->w = static_cast<uint8_t*>(p);
  if ((r = device_alloc(&p, r_bytes)) != CAI_OK) return r;
  h->rows = static_cast<uint8_t*>(p);
  if (cudaHostAlloc(&p, sizeof(uint32_t), cudaHostAllocMapped) != cudaSuccess) return CAI_ERR_NOMEM;
  h->err = static_cast<uint32_t*>(p);
  *h->err = 0;
  if (cudaHostGetDevicePointer(&p, h->err, 0) != cudaSuccess) return CAI_ERR_CUDA;
  h->d_err = static_cast<uint32_t*>(p);
  if ((r = set_up_pairs(h, w_bytes, r_bytes)) != CAI_OK) return r;
  // Scales of rows past the last, which the product reads with its whole groups.
  if (cudaMemsetAsync(h->w, 0, w_bytes, stream) != cudaSuccess ||
      cudaMemsetAsync(h->rows, 0, r_bytes, stream) != cudaSuccess)
    return CAI_ERR_CUDA;
  if ((r = pack(h, W, dtype, h->V, static_cast<long long>(h->n_vt) * h->tile, h->tile, h->w, nullptr,
                stream)) != CAI_OK)
    return r;
  return cudaStreamSynchronize(stream) == cudaSuccess ? CAI_OK : CAI_ERR_CUDA;
}

}  // namespace

extern "C" void cai_mx4_free(cai_mx4* h) {
  if (!h) return;
  int dev = 0;
  const bool moved = cudaGetDevice(&dev) == cudaSuccess && dev != h->dev;
  if (moved) cudaSetDevice(h->dev);
  cudaDeviceSynchronize();
  cudaFree(h->w);
  cudaFree(h->rows);
  if (h->err) cudaFreeHost(h->err);
  if (moved) cudaSetDevice(dev);
  cudaGetLastError();
  delete h;
}

extern "C" int cai_mx4_init(const void* W, int32_t dtype, int32_t V, int32_t H, int32_t max_rows,
                            void* stream, cai_mx4** out) {
  if (!out) return CAI_ERR_ARG;
  *out = nullptr;
  if (!W || !elem_bytes(dtype)) return CAI_ERR_ARG;
  if (V < 1 || V > (1 << 22) || H < 64 || H > 16384 || H % 64 != 0 || max_rows < 1 ||
      max_rows > 65536)
    return CAI_ERR_SHAPE;
  cai_mx4* h = new (std::nothrow) cai_mx4;
  if (!h) return CAI_ERR_NOMEM;
  h->V = V;
  h->H = H;
  h->max_rows = max_rows;
  const int r = init(h, W, dtype, static_cast<cudaStream_t>(stream));
  if (r != CAI_OK) {
    cudaGetLastError();
    cai_mx4_free(h);
    return r;
  }
  *out = h;
  return CAI_OK;
}

extern "C" int cai_mx4_update(cai_mx4* h, const void* W, int32_t dtype, void* values, void* stream) {
  int r = usable(h);
  if (r != CAI_OK) return r;
  if ((r = check_weight(h, W, dtype, values)) != CAI_OK) return r;
  return pack(h, W, dtype, h->V, static_cast<long long>(h->n_vt) * h->tile, h->tile, h->w, values,
              static_cast<cudaStream_t>(stream));
}

extern "C" int cai_mx4_logits(cai_mx4* h, const void* rows, int32_t dtype, int32_t M, void* out,
                              int32_t out_dtype, int64_t ld, void* stream) {
  int r = usable(h);
  if (r != CAI_OK) return r;
  if (!elem_bytes(dtype) || !elem_bytes(out_dtype)) return CAI_ERR_ARG;
  if (M < 0 || M > h->max_rows) return CAI_ERR_SHAPE;
  if (M == 0) return CAI_OK;
  if (!rows || !out || ld < h->V || reinterpret_cast<uintptr_t>(rows) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(out) % elem_bytes(out_dtype) != 0 || !on_device(rows, h->dev) ||
      !on_device(out, h->dev))
    return CAI_ERR_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((r = pack(h, rows, dtype, M, M, kMx4RowTile, h->rows, nullptr, s)) != CAI_OK) return r;
  Mx4Params p{};
  p.w = h->w;
  p.rows = h->rows;
  p.out = out;
  p.ld = ld;
  p.M = M;
  p.V = h->V;
  p.KB = h->KB;
  p.tile = h->tile;
  p.n_vt = h->n_vt;
  p.err = h->d_err;
  if (M > kMx4RowTile) {
    p.n_mt = (M + 2 * kMx4RowTile - 1) / (2 * kMx4RowTile);
    p.stages = h->pair_stages[out_dtype == CAI_F32];
    const long long tiles = static_cast<long long>(p.n_vt) * p.n_mt;
    const int grid = 2 * static_cast<int>(tiles < h->pairs ? tiles : h->pairs);
    const size_t smem = mx4_pair_smem_bytes(p.stages, p.tile, elem_bytes(out_dtype));
    const bool ok = out_dtype == CAI_BF16 ? launch_pairs<__nv_bfloat16>(h, p, grid, smem, s)
                                          : launch_pairs<float>(h, p, grid, smem, s);
    if (ok) return CAI_OK;
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  p.a_rows = (M + 7) / 8 * 8;
  p.a_bytes = p.a_rows * 128;
  p.stages = kMx4MaxStages;
  while (p.stages > 2 && mx4_smem_bytes(p.stages, p.a_bytes, p.tile, elem_bytes(out_dtype)) > h->smem_limit)
    --p.stages;
  const int grid = p.n_vt < h->sms ? p.n_vt : h->sms;
  const size_t smem = mx4_smem_bytes(p.stages, p.a_bytes, p.tile, elem_bytes(out_dtype));
  const bool ok = out_dtype == CAI_BF16 ? launch_product<__nv_bfloat16>(p, grid, smem, s)
                                        : launch_product<float>(p, grid, smem, s);
  if (!ok) {
    cudaGetLastError();
    return CAI_ERR_CUDA;
  }
  return CAI_OK;
}

extern "C" int cai_mx4_error_bits(const cai_mx4* h, uint32_t* bits) {
  if (!h || !bits) return CAI_ERR_ARG;
  *bits = *reinterpret_cast<volatile uint32_t*>(h->err);
  return CAI_OK;
}
