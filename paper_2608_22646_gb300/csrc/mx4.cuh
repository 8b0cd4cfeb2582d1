// An LM-head weight in microscaled 4-bit floating point (cai_mx4_*): blocks of
// 32 values along H share a power of two (E8M0), the values are E2M1.
//
//   scale of a block: 2^(floor(log2 max|x|) - 2); codes: x / scale rounded to
//   the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, larger
//   ones to 6.  logits[m, v] = sum over blocks of scale_m scale_v (codes . codes).
//
// Layout.  What one tensor-core step reads lies together in HBM as it will lie
// in shared memory: for `tile` rows and 256 values of H, the codes as rows of 128
// bytes in the 128-byte swizzle, then their scales in groups of 128 rows and 128
// values (512 bytes: row i of 32 at 16 i, its row group j at + 4 j, the four
// blocks' bytes in order), as tcgen05.cp brings them into tensor memory.  One
// bulk copy loads all of it.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>

#include "ptx.cuh"

namespace cai {

constexpr int kMx4Block = 32;          // values per scale
constexpr int kMx4K = 256;             // values of H per stage: 128 bytes of codes
constexpr int kMx4MaxTile = 224;       // vocabulary rows per tile, at most
constexpr int kMx4RowTile = 128;       // rows of the step per tile (MMA M)
constexpr int kMx4ScaleAtom = 512;     // scales of 128 rows and 128 values

// Bytes of a tile's stage.
__host__ __device__ constexpr int mx4_scale_bytes(int tile) {
  return 2 * ((tile + 127) / 128) * kMx4ScaleAtom;
}
__host__ __device__ constexpr int mx4_stage_bytes(int tile) {
  return tile * 128 + mx4_scale_bytes(tile);
}

// ------------------------------------------------------------ quantisation --

struct Mx4PackParams {
  const void* src;      // [rows, H]
  uint8_t* dst;
  __nv_bfloat16* values;  // [rows, H] or null: what the codes stand for
  long long rows;       // of src
  long long rows_pad;   // rows written: those past `rows` get zeros
  int H, KB, tile;
};

// Eight values of a row as floats.
__device__ __forceinline__ void mx4_load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void mx4_load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// Two values as E2M1 codes, the first in the low half of a byte.
__device__ __forceinline__ uint32_t mx4_code2(float lo, float hi) {
  uint16_t r;
  asm("{\n\t.reg .b8 t;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\t"
      "cvt.u16.u8 %0, t;\n\t}"
      : "=h"(r)
      : "f"(hi), "f"(lo));
  return r;
}
// The two values that a byte of codes stands for.
__device__ __forceinline__ float2 mx4_value2(uint32_t byte) {
  uint32_t h;
  asm("{\n\t.reg .b8 t;\n\t"
      "cvt.u8.u32 t, %1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, t;\n\t}"
      : "=r"(h)
      : "r"(byte));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// 16 lanes take 128 values of a row, eight each: four lanes a block.
template <typename T>
__global__ void __launch_bounds__(256) mx4_pack_kernel(const Mx4PackParams p) {
  grid_launch_dependents();
  const int lane = threadIdx.x & 31, sub = lane & 15;
  const int per_row = 2 * p.KB;  // groups of 128 values
  const long long n = p.rows_pad * per_row;
  const long long step = static_cast<long long>(gridDim.x) * (blockDim.x / 16);
  const int stage = mx4_stage_bytes(p.tile), groups = (p.tile + 127) / 128;
  for (long long q = blockIdx.x * (blockDim.x / 16) + (threadIdx.x >> 4) - ((lane >> 4) & 1);; q += step) {
    // q counts for the warp's first half; both halves stay together.
    const long long item = q + (lane >> 4);
    if (q >= n) break;
    const long long row = item / per_row;
    const int k128 = static_cast<int>(item - row * per_row);
    const int k = k128 * 128 + sub * 8;
    float x[8] = {};
    if (item < n && row < p.rows && k < p.H) mx4_load8(static_cast<const T*>(p.src) + row * p.H + k, x);
    float high = 0.0f;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      high = fmaxf(high, fabsf(x[i]));
      finite &= fabsf(x[i]) <= 3.402823466e38f;
    }
    high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, 1));
    high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, 2));
    const uint32_t ok = __ballot_sync(0xffffffffu, finite);
    // The scale's exponent, biased: that of the largest value less 2; 255 (no
    // number) where a value is none.
    const int e = static_cast<int>(__float_as_uint(high) >> 23);
    uint32_t code = e > 2 ? e - 2 : 0;
    if (((ok >> (lane & 28)) & 15u) != 15u) code = 255;
    const float inv = __uint_as_float(code == 255 ? 0u : (254u - code) << 23);
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) packed |= mx4_code2(x[2 * i] * inv, x[2 * i + 1] * inv) << (8 * i);
    uint32_t scales = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      scales |= __shfl_sync(0xffffffffu, code, (lane & 16) + 4 * j) << (8 * j);
    if (item < n) {
      const long long t = row / p.tile;
      const int r = static_cast<int>(row - t * p.tile);
      uint8_t* base = p.dst + (t * p.KB + (k128 >> 1)) * stage;
      const int chunk = (k128 & 1) * 4 + (sub >> 2);
      *reinterpret_cast<uint32_t*>(base + r * 128 + ((chunk ^ (r & 7)) << 4) + (sub & 3) * 4) = packed;
      if (sub == 0)
        *reinterpret_cast<uint32_t*>(base + p.tile * 128 +
                                     ((k128 & 1) * groups + (r >> 7)) * kMx4ScaleAtom +
                                     (r & 31) * 16 + ((r >> 5) & 3) * 4) = scales;
      if (p.values && row < p.rows && k < p.H) {
        const float scale = __uint_as_float(code == 255 ? 0x7fc00000u : code ? code << 23 : 0x00400000u);
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = mx4_value2((packed >> (8 * i)) & 255u);
          const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
          v[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(p.values + row * p.H + k) = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  }
}

// ----------------------------------------------------------------- product --

// Instruction descriptor of tcgen05.mma kind::mxf4: A and B E2M1 (bits 7-9 and
// 10-11 = 1), K-major, N >> 3 in bits 17-22, scales E8M0 (bit 23), M >> 7 in bits
// 27-28; which half of a scale column's four bytes holds this step's two scales
// in bits 4-5 (B) and 29-30 (A).
__host__ __device__ constexpr uint32_t idesc_mxf4(uint32_t M, uint32_t N, uint32_t half) {
  return ((2 * half) << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) |
         ((M >> 7) << 27) | ((2 * half) << 29);
}

// D[tmem] (+)= (A . scales) (B . scales)^T over 64 values, issued by one thread.
__device__ __forceinline__ void mma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                         uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
          d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}

// 32 rows of 16 bytes from shared memory into four columns of all four lane
// quarters; in order with the MMAs of the same thread.
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t sdesc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}

// Descriptor of a scale group: no swizzle, 8 rows of 16 bytes 128 bytes apart.
__device__ __forceinline__ uint64_t sdesc_scales(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(1u) << 16) |
         (static_cast<uint64_t>(128u >> 4) << 32) | (static_cast<uint64_t>(1u) << 46);
}

constexpr int kMx4EpiWarps = 4;
constexpr int kMx4Threads = 64 + 32 * kMx4EpiWarps;
constexpr uint32_t kMx4TmemCols = 512;
constexpr uint32_t kMx4ScaleCol = 2 * kMx4MaxTile;  // scales follow the two accumulators
constexpr uint32_t kMx4ScaleCols = 24;              // of one stage: 8 of the rows, 16 of W
constexpr int kMx4MaxStages = 8;
constexpr int kMx4EpiPitch = 32 * 4 + 16;           // bytes between staged rows

struct Mx4Params {
  const uint8_t* w;      // packed weight
  const uint8_t* rows;   // packed rows
  void* out;             // [M, V], ld apart
  long long ld;
  int M, V, KB, tile;
  int n_vt, n_mt;        // tiles along V, along M
  int a_rows;            // rows of a row tile that are loaded (a multiple of 8)
  int a_bytes;           // room for their codes (a multiple of 1 KiB)
  int stages;
  uint32_t* err;
};

__host__ __device__ inline int mx4_smem_stage(int a_bytes, int tile) {
  return a_bytes + mx4_scale_bytes(kMx4RowTile) + mx4_stage_bytes(tile);
}
// The MMA reads 128 rows of A whatever was loaded; past the last stage's there
// is at least that much allocated.
__host__ inline size_t mx4_smem_bytes(int stages, int a_bytes, int tile) {
  return 1024 + static_cast<size_t>(stages) * mx4_smem_stage(a_bytes, tile) + 16384 +
         kMx4EpiWarps * 32 * kMx4EpiPitch;
}

struct Mx4Ring {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int n) {
    if (++slot == n) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// Waits, with a limit, for copies or MMAs in flight on an abort path.
__device__ __forceinline__ void mx4_drain(uint64_t* bar, uint32_t parity, uint32_t* err) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity))
    if (global_timer_ns() - t0 > kWaitLimitNs) {
      atomicOr_system(err, kErrDrain);
      return;
    }
}

template <typename T>
__device__ __forceinline__ T mx4_out(float x);
template <>
__device__ __forceinline__ float mx4_out<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ __nv_bfloat16 mx4_out<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}

// One CTA per SM; each takes tiles of 128 rows by `tile` vocabulary rows, those
// that share W next to each other in time.  Warp 0 copies stages, warp 1 issues
// the scales' copies and the MMAs, warps 2-5 write the accumulators out through
// shared memory, so that a row's logits leave as whole 32-byte sectors.
template <typename T>
__global__ void __launch_bounds__(kMx4Threads, 1) mx4_logits_kernel(const Mx4Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMx4MaxStages], empty[kMx4MaxStages], accf[2], acce[2], drain;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sstage = mx4_smem_stage(p.a_bytes, p.tile);
  const int b_bytes = mx4_stage_bytes(p.tile);
  uint8_t* staging = smem + static_cast<size_t>(p.stages) * sstage + 16384;
  const int tiles = p.n_vt * p.n_mt;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&accf[a], 1);
      mbar_init(&acce[a], kMx4EpiWarps);
    }
    mbar_init(&drain, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_slot, kMx4TmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // Every role: the rows' codes come from the kernel before, and the bounded
  // waits must not include it.
  grid_dependency_wait();

  if (warp == 0) {
    const uint64_t pol_w = p.n_mt > 1 ? policy_evict_last() : policy_evict_first();
    const uint64_t pol_r = policy_evict_last();
    const bool leader = elect_one();
    const int a_codes = p.a_rows * 128;
    constexpr int kRowStage = mx4_stage_bytes(kMx4RowTile);
    Mx4Ring r;
    int issued = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      const int vt = t / p.n_mt, mt = t - vt * p.n_mt;
      const uint8_t* wsrc = p.w + static_cast<size_t>(vt) * p.KB * b_bytes;
      const uint8_t* rsrc = p.rows + static_cast<size_t>(mt) * p.KB * kRowStage;
      for (int kb = 0; kb < p.KB; ++kb) {
        ok = ok && mbar_wait(&empty[r.slot], r.phase ^ 1u, &abort_flag, p.err, kErrWaitEmpty);
        if (leader && ok) {
          uint8_t* s = smem + static_cast<size_t>(r.slot) * sstage;
          mbar_arrive_expect_tx(&full[r.slot], b_bytes + a_codes + mx4_scale_bytes(kMx4RowTile));
          bulk_load(s + p.a_bytes + mx4_scale_bytes(kMx4RowTile), wsrc + static_cast<size_t>(kb) * b_bytes,
                    b_bytes, &full[r.slot], pol_w);
          const uint8_t* a = rsrc + static_cast<size_t>(kb) * kRowStage;
          bulk_load(s, a, a_codes, &full[r.slot], pol_r);
          bulk_load(s + p.a_bytes, a + kMx4RowTile * 128, mx4_scale_bytes(kMx4RowTile), &full[r.slot], pol_r);
        }
        __syncwarp();
        issued += ok ? 1 : 0;
        r.next(p.stages);
      }
      ok = __all_sync(0xffffffffu, ok);
    }
    if (leader && !ok)
      for (int i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i)
        mx4_drain(&full[i % p.stages], static_cast<uint32_t>((i / p.stages) & 1), p.err);
    __syncwarp();
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint32_t groups = (p.tile + 127) / 128;
    const uint32_t id0 = idesc_mxf4(kMx4RowTile, p.tile, 0), id1 = idesc_mxf4(kMx4RowTile, p.tile, 1);
    Mx4Ring r, acc;
    uint32_t turn = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      ok = __all_sync(0xffffffffu, mbar_wait(&acce[acc.slot], acc.phase ^ 1u, &abort_flag, p.err, kErrWaitAccEmpty));
      if (!ok) break;
      tc_fence_after();
      const uint32_t d = tmem + acc.slot * kMx4MaxTile;
      for (int kb = 0; kb < p.KB; ++kb) {
        ok = ok && mbar_wait(&full[r.slot], r.phase, &abort_flag, p.err, kErrWaitFull);
        tc_fence_after();
        if (leader && ok) {
          const uint32_t a = smem_addr(smem) + r.slot * sstage;
          const uint32_t as = a + p.a_bytes;
          const uint32_t b = as + mx4_scale_bytes(kMx4RowTile);
          const uint32_t bs = b + p.tile * 128;
          const uint32_t sf = tmem + kMx4ScaleCol + (turn & 1u) * kMx4ScaleCols;
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {
            tmem_cp_scales(sf + 4 * h, sdesc_scales(as + h * kMx4ScaleAtom));
            for (uint32_t g = 0; g < groups; ++g)
              tmem_cp_scales(sf + 8 + 8 * h + 4 * g, sdesc_scales(bs + (h * groups + g) * kMx4ScaleAtom));
          }
          const uint64_t ad = sdesc_k_sw128(a), bd = sdesc_k_sw128(b);
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)
            mma_mxf4(d, ad + 2 * j, bd + 2 * j, j & 1 ? id1 : id0, sf + 4 * (j >> 1),
                     sf + 8 + 8 * (j >> 1), (kb | j) != 0 ? 1u : 0u);
          mma_commit(&empty[r.slot]);
        }
        __syncwarp();
        ++turn;
        r.next(p.stages);
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (leader) mma_commit(&accf[acc.slot]);
      __syncwarp();
      acc.next(2);
    }
    if (leader && !ok) {
      mma_commit(&drain);
      mx4_drain(&drain, 0, p.err);
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;
    uint8_t* mine = staging + quarter * 32 * kMx4EpiPitch;
    constexpr int kPer16 = 16 / sizeof(T);           // values of a 16-byte store
    constexpr int kLanes = 32 / kPer16;              // lanes of a row's 32 values
    const bool aligned = (reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(p.ld * sizeof(T))) % 16 == 0;
    Mx4Ring acc;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
      if (!mbar_wait(&accf[acc.slot], acc.phase, &abort_flag, p.err, kErrWaitAccFull)) break;
      tc_fence_after();
      const int vt = t / p.n_mt, mt = t - vt * p.n_mt;
      const int row0 = mt * kMx4RowTile + quarter * 32;
      const int n_rows = min(32, p.M - row0);  // of this warp; may be 0 or less
      const int v0 = vt * p.tile;
      const int n_v = min(p.tile, p.V - v0);
      if (n_rows > 0) {
        const uint32_t src = tmem + acc.slot * kMx4MaxTile + (static_cast<uint32_t>(quarter * 32) << 16);
        T* out = static_cast<T*>(p.out) + static_cast<long long>(row0) * p.ld + v0;
        for (int c = 0; c < n_v; c += 32) {
          uint32_t x[32];
          tmem_ld_32cols(src + c, x);
          tmem_ld_wait();
          T* st = reinterpret_cast<T*>(mine + lane * kMx4EpiPitch);
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(x[8 * i + 2 * j]),
                                                               __uint_as_float(x[8 * i + 2 * j + 1]));
                w[j] = *reinterpret_cast<const uint32_t*>(&b);
              }
              reinterpret_cast<uint4*>(st)[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              reinterpret_cast<uint4*>(st)[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
          }
          __syncwarp();
          const int left = n_v - c;
          if (aligned && left >= 32) {
#pragma unroll
            for (int i = 0; i < kLanes; ++i) {
              const int rr = i * (32 / kLanes) + lane / kLanes, q = lane % kLanes;
              if (rr < n_rows)
                *reinterpret_cast<uint4*>(out + static_cast<long long>(rr) * p.ld + c + q * kPer16) =
                    reinterpret_cast<const uint4*>(mine + rr * kMx4EpiPitch)[q];
            }
          } else if (lane < left) {
            for (int rr = 0; rr < n_rows; ++rr)
              out[static_cast<long long>(rr) * p.ld + c + lane] =
                  reinterpret_cast<const T*>(mine + rr * kMx4EpiPitch)[lane];
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acce[acc.slot]);
      acc.next(2);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kMx4TmemCols);
  }
}

}  // namespace cai
