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

constexpr int kMx4K = 256;             // values of H per stage: 128 bytes of codes
constexpr int kMx4MaxTile = 208;       // vocabulary rows per tile, at most
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

// Eight values of a row, as they lie in memory and as floats.
template <typename T>
struct Mx4Eight {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                   : "l"(reinterpret_cast<const uint4*>(p) + i));
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) v[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = sizeof(T) == 4 ? __uint_as_float(w[i])
                            : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  // The biased exponent of the largest magnitude, 255 where a value is not finite.
  // Magnitudes compare as whole numbers, infinities and NaN above all others.
  __device__ __forceinline__ uint32_t exponent() const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
    if (sizeof(T) == 4) {
      uint32_t m = w[0] & 0x7fffffffu;
#pragma unroll
      for (int i = 1; i < 8; ++i) m = max(m, w[sizeof(T) == 4 ? i : 0] & 0x7fffffffu);
      return m >> 23;
    }
    uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    return max(m >> 16, m & 0xffffu) >> 7;
  }
};

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

// Where a group of 128 values of a row lies: in the source, and in the packed
// tiles.  Moves on by a fixed number of groups without a division.
struct Mx4Place {
  uint32_t row, k;  // k: which group of the row
  uint32_t t, r;    // tile, row in it
  __device__ __forceinline__ Mx4Place(uint32_t item, uint32_t per_row, uint32_t tile) {
    row = item / per_row;
    k = item - row * per_row;
    t = row / tile;
    r = row - t * tile;
  }
  __device__ __forceinline__ void move(const Mx4Place& by, uint32_t per_row, uint32_t tile) {
    k += by.k;
    const uint32_t wrap = k >= per_row;
    k -= wrap ? per_row : 0;
    row += by.row + wrap;
    r += by.r + wrap;
    t += by.t;
    if (r >= tile) {
      r -= tile;
      ++t;
    }
  }
};

// Eight lanes take a group of 128 values: eight values in each half, of which four
// lanes hold a block.  Bound by its bytes (126464 x 4096 bf16 with values: 373 us,
// 344 at the copy's rate; without 239, of 195; float32 with values 516, of 497).
// Sixteen lanes to a group, positions divided out and a separate test for numbers
// cost 210 instructions for eight values, and 474 us.  Many CTAs of few turns keep
// more loads in flight than turns of several groups do: 256 CTAs to an SM 373 us,
// 64 382, 1000 402; with four groups a turn on 8 404, on 32 387.
template <typename T>
__global__ void __launch_bounds__(256) mx4_pack_kernel(const Mx4PackParams p) {
  grid_launch_dependents();
  constexpr uint32_t kItems = 256 / 8;  // of a CTA
  const int lane = threadIdx.x & 31, sub = lane & 7;
  const uint32_t per_row = 2 * p.KB, tile = p.tile;
  // At most 2^22 rows of 128 groups, and some.
  const uint32_t n = static_cast<uint32_t>(p.rows_pad) * per_row;
  const uint32_t step = gridDim.x * kItems;
  const uint32_t stage = mx4_stage_bytes(p.tile), groups = (tile + 127) / 128;
  uint32_t q = blockIdx.x * kItems + (threadIdx.x >> 3);
  const Mx4Place by(step, per_row, tile);
  Mx4Place at(q, per_row, tile);
#pragma unroll 1
  for (; (q & ~3u) < n; q += step) {  // the same in the whole warp
    const int k = static_cast<int>(at.k) * 128 + sub * 8;
    const bool there = q < n && at.row < p.rows;
    const T* src = static_cast<const T*>(p.src) + static_cast<long long>(at.row) * p.H + k;
    Mx4Eight<T> in[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (there && k + 64 * h < p.H)
        in[h].load(src + 64 * h);
      else
        in[h].zero();
    uint32_t code[2], packed[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t e = in[h].exponent();
      e = max(e, __shfl_xor_sync(0xffffffffu, e, 1));
      e = max(e, __shfl_xor_sync(0xffffffffu, e, 2));
      // The scale's exponent, biased: that of the largest value less 2; 255 (no
      // number) where a value is none.
      code[h] = e == 255 ? 255u : max(e, 2u) - 2u;
      const float inv = __uint_as_float(e == 255 ? 0u : (254u - code[h]) << 23);
      float x[8];
      in[h].floats(x);
      packed[h] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = __fmul2_rn(make_float2(x[2 * i], x[2 * i + 1]), make_float2(inv, inv));
        packed[h] |= mx4_code2(y.x, y.y) << (8 * i);
      }
    }
    uint32_t scales = code[0] | code[1] << 16;
    scales |= __shfl_xor_sync(0xffffffffu, scales, 4) << 8;  // whole in the first four lanes
    if (q < n) {
      uint8_t* base = p.dst + (static_cast<size_t>(at.t) * p.KB + (at.k >> 1)) * stage;
      const uint32_t half = at.k & 1, chunk = (half * 4 + (sub >> 2)) ^ (at.r & 7);
      uint8_t* codes = base + at.r * 128 + (sub & 3) * 4;
      *reinterpret_cast<uint32_t*>(codes + (chunk << 4)) = packed[0];
      *reinterpret_cast<uint32_t*>(codes + ((chunk ^ 2) << 4)) = packed[1];
      if (sub == 0)
        *reinterpret_cast<uint32_t*>(base + tile * 128 + (half * groups + (at.r >> 7)) * kMx4ScaleAtom +
                                     (at.r & 31) * 16 + ((at.r >> 5) & 3) * 4) = scales;
    }
    if (there && p.values) {
      __nv_bfloat16* out = p.values + static_cast<long long>(at.row) * p.H + k;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (k + 64 * h >= p.H) break;
        const float scale =
            __uint_as_float(code[h] == 255 ? 0x7fc00000u : code[h] ? code[h] << 23 : 0x00400000u);
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 y = __fmul2_rn(mx4_value2((packed[h] >> (8 * i)) & 255u), make_float2(scale, scale));
          const __nv_bfloat162 b = __floats2bfloat162_rn(y.x, y.y);
          v[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        __stcs(reinterpret_cast<uint4*>(out + 64 * h), make_uint4(v[0], v[1], v[2], v[3]));
      }
    }
    at.move(by, per_row, tile);
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
// kPair: over a CTA pair, by the even CTA (see mma_bf16_pair): each CTA has its
// rows' scales in its tensor memory, and all of W's.
template <bool kPair>
__device__ __forceinline__ void mma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                         uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
  if constexpr (kPair)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// 32 rows of 16 bytes from shared memory into four columns of all four lane
// quarters (kPair: in both CTAs, each from its own); in order with the MMAs of the
// same thread.
template <bool kPair>
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t sdesc) {
  if constexpr (kPair)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}

// Descriptor of a scale group: no swizzle, 8 rows of 16 bytes 128 bytes apart.
__device__ __forceinline__ uint64_t sdesc_scales(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(1u) << 16) |
         (static_cast<uint64_t>(128u >> 4) << 32) | (static_cast<uint64_t>(1u) << 46);
}

constexpr int kMx4EpiWarps = 8;  // two for each quarter of the rows
constexpr int kMx4Threads = 64 + 32 * kMx4EpiWarps;
constexpr uint32_t kMx4TmemCols = 512;
constexpr uint32_t kMx4AccCol = 224;                // columns between the two accumulators
constexpr uint32_t kMx4ScaleCol = kMx4AccCol + kMx4MaxTile;  // scales follow them
constexpr uint32_t kMx4ScaleCols = 24;              // of one stage: 8 of the rows, 16 of W
constexpr uint32_t kMx4ScaleBufs = 3;
static_assert(kMx4ScaleCol + kMx4ScaleBufs * kMx4ScaleCols <= kMx4TmemCols, "tensor memory");
constexpr int kMx4MaxStages = 8;

// Bytes between the rows of 32 values that a warp writes out through shared memory.
__host__ __device__ constexpr int mx4_pitch(int elem) { return 32 * elem + 16; }

struct Mx4Params {
  const uint8_t* w;      // packed weight
  const uint8_t* rows;   // packed rows
  void* out;             // [M, V], ld apart
  long long ld;
  int M, V, KB, tile;
  int n_vt;              // tiles along V
  int n_mt;              // tiles of 256 rows along M (the pair kernel)
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
__host__ inline size_t mx4_smem_bytes(int stages, int a_bytes, int tile, int elem) {
  return 1024 + static_cast<size_t>(stages) * mx4_smem_stage(a_bytes, tile) + 16384 +
         kMx4EpiWarps * 32 * mx4_pitch(elem);
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

// A warp writes its 32 rows by n_v columns of an accumulator (tensor memory `src`,
// its lanes) out through shared memory `mine`, so that a row's logits leave as
// whole 32-byte sectors.  out: the first row's first column; n_rows may be 0 or
// less.  aligned: out's rows begin at multiples of 16 bytes.  part: which of the two
// warps that share the rows this is; they take 32 columns in turn.
template <typename T>
__device__ __forceinline__ void mx4_store_tile(uint32_t src, uint8_t* mine, T* out, long long ld,
                                               int n_rows, int n_v, bool aligned, int part) {
  constexpr int kPitch = mx4_pitch(sizeof(T));
  constexpr int kPer16 = 16 / sizeof(T);           // values of a 16-byte store
  constexpr int kLanes = 32 / kPer16;              // lanes of a row's 32 values
  const int lane = threadIdx.x & 31;
  if (n_rows <= 0) return;
#pragma unroll 1
  for (int c = 32 * part; c < n_v; c += 64) {
    uint32_t x[32];
    tmem_ld_32cols(src + c, x);
    tmem_ld_wait();
    uint4* st = reinterpret_cast<uint4*>(mine + lane * kPitch);
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
        st[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) st[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
    __syncwarp();
    const int left = n_v - c;
    if (aligned && left >= 32) {
#pragma unroll
      for (int i = 0; i < kLanes; ++i) {
        const int rr = i * (32 / kLanes) + lane / kLanes, q = lane % kLanes;
        if (rr < n_rows)
          __stcs(reinterpret_cast<uint4*>(out + static_cast<long long>(rr) * ld + c + q * kPer16),
                 reinterpret_cast<const uint4*>(mine + rr * kPitch)[q]);
      }
    } else if (lane < left) {
      T* to = out + c + lane;
      const int n = min(n_rows, 32);
#pragma unroll 8
      for (int rr = 0; rr < n; ++rr, to += ld)
        *to = reinterpret_cast<const T*>(mine + rr * kPitch)[lane];
    }
    __syncwarp();
  }
}

// A stage's scales into tensor memory (columns sf), and its four MMAs, issued by
// one thread.  as, bs: the scales of the rows and of W; a, b: their codes.
template <bool kPair>
__device__ __forceinline__ void mx4_issue_scales(uint32_t sf, uint32_t as, uint32_t bs, uint32_t groups) {
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h) {
    tmem_cp_scales<kPair>(sf + 4 * h, sdesc_scales(as + h * kMx4ScaleAtom));
    for (uint32_t g = 0; g < groups; ++g)
      tmem_cp_scales<kPair>(sf + 8 + 8 * h + 4 * g, sdesc_scales(bs + (h * groups + g) * kMx4ScaleAtom));
  }
}
template <bool kPair>
__device__ __forceinline__ void mx4_issue_mmas(uint32_t d, uint32_t a, uint32_t b, uint32_t sf, uint32_t id0,
                                               uint32_t id1, bool first) {
  const uint64_t ad = sdesc_k_sw128(a), bd = sdesc_k_sw128(b);
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    mma_mxf4<kPair>(d, ad + 2 * j, bd + 2 * j, j & 1 ? id1 : id0, sf + 4 * (j >> 1), sf + 8 + 8 * (j >> 1),
                    first && j == 0 ? 0u : 1u);
}

// The MMA warp's loop: n_tiles tiles of p.KB stages.  A stage's scales go to one of
// three places in turn (2048 x 126464 x 4096: one place 451 us, two 416, three 409;
// copied a stage ahead of their MMAs, 515: the MMAs then wait for the next stage's
// bytes too).  The six copies of a stage are what keeps a step from its MMAs' time:
// without them 308 us, without the MMAs 364.
template <bool kPair>
__device__ __forceinline__ bool mx4_issue_all(const Mx4Params& p, int n_tiles, uint32_t smem, int sstage,
                                              uint32_t as_at, uint32_t b_at, uint32_t bs_at, uint32_t tmem,
                                              uint64_t* full, uint64_t* empty, uint64_t* accf, uint64_t* acce,
                                              volatile int* abort_flag, bool leader) {
  constexpr uint32_t kRows = (kPair ? 2 : 1) * kMx4RowTile;
  const uint32_t groups = (p.tile + 127) / 128;
  const uint32_t id0 = idesc_mxf4(kRows, p.tile, 0), id1 = idesc_mxf4(kRows, p.tile, 1);
  const auto wait = [&](uint64_t* bar, uint32_t phase, uint32_t site) {
    return __all_sync(0xffffffffu, kPair ? mbar_wait_cluster(bar, phase, abort_flag, p.err, site)
                                         : mbar_wait(bar, phase, abort_flag, p.err, site));
  };
  Mx4Ring r, acc;
  uint32_t buf = 0;
  for (int t = 0; t < n_tiles; ++t) {
    if (!wait(&acce[acc.slot], acc.phase ^ 1u, kErrWaitAccEmpty)) return false;
    tc_fence_after();
    for (int kb = 0; kb < p.KB; ++kb) {
      if (!wait(&full[r.slot], r.phase, kErrWaitFull)) return false;
      tc_fence_after();
      if (leader) {
        const uint32_t s = smem + r.slot * sstage;
        const uint32_t sf = tmem + kMx4ScaleCol + buf * kMx4ScaleCols;
        mx4_issue_scales<kPair>(sf, s + as_at, s + bs_at, groups);
        mx4_issue_mmas<kPair>(tmem + acc.slot * kMx4AccCol, s, s + b_at, sf, id0, id1, kb == 0);
        if (kPair)
          mma_commit_pair(&empty[r.slot], 0x3);
        else
          mma_commit(&empty[r.slot]);
      }
      __syncwarp();
      r.next(p.stages);
      if (++buf == kMx4ScaleBufs) buf = 0;
    }
    if (leader) {
      if (kPair)
        mma_commit_pair(&accf[acc.slot], 0x3);
      else
        mma_commit(&accf[acc.slot]);
    }
    __syncwarp();
    acc.next(2);
  }
  return true;
}

// Up to 128 rows: the rows' codes as A (M = 128, of which a step owns few), a tile
// of the vocabulary as B, one CTA on an SM over tiles; two accumulators, so that a
// tile leaves while the next is summed.  Bound by W's bytes: 1 row, V = 126464, H =
// 4096, 47 us with the packing launch, 41 at the copy's rate of 275 MB; 128 rows 53.
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
  const int tiles = p.n_vt;
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
    const uint64_t pol_w = policy_evict_first();
    const uint64_t pol_r = policy_evict_last();
    const bool leader = elect_one();
    const int a_codes = p.a_rows * 128;
    constexpr int kRowStage = mx4_stage_bytes(kMx4RowTile);
    Mx4Ring r;
    int issued = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      const uint8_t* wsrc = p.w + static_cast<size_t>(t) * p.KB * b_bytes;
      for (int kb = 0; kb < p.KB; ++kb) {
        ok = ok && mbar_wait(&empty[r.slot], r.phase ^ 1u, &abort_flag, p.err, kErrWaitEmpty);
        if (leader && ok) {
          uint8_t* s = smem + static_cast<size_t>(r.slot) * sstage;
          mbar_arrive_expect_tx(&full[r.slot], b_bytes + a_codes + mx4_scale_bytes(kMx4RowTile));
          bulk_load(s + p.a_bytes + mx4_scale_bytes(kMx4RowTile), wsrc + static_cast<size_t>(kb) * b_bytes,
                    b_bytes, &full[r.slot], pol_w);
          const uint8_t* a = p.rows + static_cast<size_t>(kb) * kRowStage;
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
    const int mine = static_cast<int>(blockIdx.x) < tiles ? (tiles - 1 - blockIdx.x) / gridDim.x + 1 : 0;
    const uint32_t as_at = p.a_bytes, b_at = as_at + mx4_scale_bytes(kMx4RowTile);
    const bool ok = mx4_issue_all<false>(p, mine, smem_addr(smem), sstage, as_at, b_at, b_at + p.tile * 128, tmem,
                                         full, empty, accf, acce, &abort_flag, leader);
    if (leader && !ok) {
      mma_commit(&drain);
      mx4_drain(&drain, 0, p.err);
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    uint8_t* mine = staging + (warp - 2) * 32 * mx4_pitch(sizeof(T));
    const bool aligned = (reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(p.ld * sizeof(T))) % 16 == 0;
    Mx4Ring acc;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
      if (!mbar_wait(&accf[acc.slot], acc.phase, &abort_flag, p.err, kErrWaitAccFull)) break;
      tc_fence_after();
      const int row0 = quarter * 32, v0 = t * p.tile;
      mx4_store_tile<T>(tmem + acc.slot * kMx4AccCol + (static_cast<uint32_t>(quarter * 32) << 16), mine,
                        static_cast<T*>(p.out) + static_cast<long long>(row0) * p.ld + v0, p.ld,
                        p.M - row0, min(p.tile, p.V - v0), aligned, part);
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

// More than 128 rows: CTA pairs (cta_group::2) on tiles of 256 rows, each CTA with
// its 128 rows and half of the tile's W.  One CTA on 128 rows takes 46 KiB into its
// shared memory for MMAs of 0.22 us, more than an SM's share of L2 gives (2048 x
// 126464 x 4096: 105 KB/us, 459 us); a pair's CTA takes 32 KiB for as much (409 to
// 421, the tensor pipe busy 51 % of the time; bound by the scales' copies, which
// take turns with the MMAs).  The packed weight and rows are seen as rows of 128
// bytes for the copies, which complete on the even CTA's barriers.
struct Mx4PairMaps {
  CUtensorMap rows, w, scales;  // boxes: a row tile's stage, half a tile's codes, its scales
};

__host__ __device__ inline int mx4_pair_stage(int tile) {
  return mx4_stage_bytes(kMx4RowTile) + tile / 2 * 128 + mx4_scale_bytes(tile);
}
__host__ inline size_t mx4_pair_smem_bytes(int stages, int tile, int elem) {
  return 1024 + static_cast<size_t>(stages) * mx4_pair_stage(tile) + kMx4EpiWarps * 32 * mx4_pitch(elem);
}

template <typename T>
__global__ void __launch_bounds__(kMx4Threads, 1)
    mx4_logits_pair_kernel(const __grid_constant__ Mx4PairMaps maps, const Mx4Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMx4MaxStages], empty[kMx4MaxStages], accf[2], acce[2], drain;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int sstage = mx4_pair_stage(p.tile);
  constexpr int kRowStage = mx4_stage_bytes(kMx4RowTile);
  uint8_t* staging = smem + static_cast<size_t>(p.stages) * sstage;
  const int tiles = p.n_vt * p.n_mt;  // of 256 rows
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&accf[a], 1);
      mbar_init(&acce[a], 2 * kMx4EpiWarps);
    }
    mbar_init(&drain, 1);
    abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&maps.rows);
    prefetch_tmap(&maps.w);
    prefetch_tmap(&maps.scales);
  }
  if (warp == 1) {
    tmem_alloc_pair(&tmem_slot, kMx4TmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // barriers of both CTAs initialised, tensor memory allocated
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  grid_dependency_wait();  // every role, as in the kernel above

  if (warp == 0) {
    const uint64_t pol = policy_evict_last();
    const uint32_t full0 = mapa_shared(full, 0);  // the even CTA's barriers
    const bool leader = elect_one();
    const int half = p.tile / 2, w_rows = p.tile + mx4_scale_bytes(p.tile) / 128;
    const uint32_t tx = 2u * static_cast<uint32_t>(sstage);  // of both CTAs
    Mx4Ring r;
    int issued = 0;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs) {
      const int vt = t / p.n_mt, mt = t - vt * p.n_mt;
      const int w0 = vt * p.KB * w_rows, r0 = (2 * mt + static_cast<int>(rank)) * p.KB * (kRowStage / 128);
      for (int kb = 0; kb < p.KB; ++kb) {
        ok = ok && mbar_wait(&empty[r.slot], r.phase ^ 1u, &abort_flag, p.err, kErrWaitEmpty);
        if (leader && ok) {
          uint8_t* s = smem + static_cast<size_t>(r.slot) * sstage;
          const uint32_t bar = full0 + static_cast<uint32_t>(r.slot * 8);
          // The even CTA arms the stage for both; a copy of the odd one that
          // completes first leaves the phase open until then.
          if (rank == 0) mbar_arrive_expect_tx(&full[r.slot], tx);
          const int w = w0 + kb * w_rows;
          tma_load_2d_pair(s, &maps.rows, bar, 0, r0 + kb * (kRowStage / 128), pol);
          tma_load_2d_pair(s + kRowStage, &maps.w, bar, 0, w + static_cast<int>(rank) * half, pol);
          tma_load_2d_pair(s + kRowStage + half * 128, &maps.scales, bar, 0, w + p.tile, pol);
        }
        __syncwarp();
        issued += ok ? 1 : 0;
        r.next(p.stages);
      }
      ok = __all_sync(0xffffffffu, ok);
    }
    if (leader && !ok && rank == 0)
      for (int i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i)
        mx4_drain(&full[i % p.stages], static_cast<uint32_t>((i / p.stages) & 1), p.err);
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const bool leader = elect_one();
      const int mine = pair < tiles ? (tiles - 1 - pair) / pairs + 1 : 0;
      const bool ok = mx4_issue_all<true>(p, mine, smem_addr(smem), sstage, kMx4RowTile * 128, kRowStage,
                                          kRowStage + p.tile / 2 * 128, tmem, full, empty, accf, acce,
                                          &abort_flag, leader);
      if (leader && !ok) {
        mma_commit_pair(&drain, 0x1);
        mx4_drain(&drain, 0, p.err);
      }
      __syncwarp();
    }
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    uint8_t* mine = staging + (warp - 2) * 32 * mx4_pitch(sizeof(T));
    const uint32_t acce0 = mapa_shared(acce, 0);
    const bool aligned = (reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(p.ld * sizeof(T))) % 16 == 0;
    Mx4Ring acc;
    for (int t = pair; t < tiles; t += pairs) {
      if (!mbar_wait(&accf[acc.slot], acc.phase, &abort_flag, p.err, kErrWaitAccFull)) break;
      tc_fence_after();
      const int vt = t / p.n_mt, mt = t - vt * p.n_mt;
      const int row0 = (2 * mt + static_cast<int>(rank)) * kMx4RowTile + quarter * 32;
      const int v0 = vt * p.tile;
      mx4_store_tile<T>(tmem + acc.slot * kMx4AccCol + (static_cast<uint32_t>(quarter * 32) << 16), mine,
                        static_cast<T*>(p.out) + static_cast<long long>(row0) * p.ld + v0, p.ld,
                        p.M - row0, min(p.tile, p.V - v0), aligned, part);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(acce0 + static_cast<uint32_t>(acc.slot * 8));
      acc.next(2);
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // no CTA leaves while the pair's MMAs or arrivals may touch it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kMx4TmemCols);
  }
}

}  // namespace cai
