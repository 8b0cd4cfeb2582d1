// AdamW over many tensors, with states in 32 or in 8 bits (cai_adamw_step).  Every
// operation is rounded once (no fused multiply-add), so that a state's code does
// not depend on how a compiler contracts: include/cai.h has the formulas.  (The
// update's quotient alone, which no state depends on, is a product with a reciprocal.)
//
// 8 bits: m and sqrt(v) as E4M3 in blocks of 32 under a power of two.  With
// beta2 = 0.999 a v moves by a thousandth of itself a step, E4M3's step is an eighth:
// rounded to nearest it would never move.  So the last place is rounded up with
// the probability of what is cut off; where that makes 0 of a number, 1 is kept,
// since a root of 0 under an m that is not would divide by eps.  But an m that its
// gradient does not bring to the smallest code may become 0 once it has a root: kept at
// 1 it would hold its sign for as long as its block has larger numbers, while its root
// decays, and in time move a parameter whose gradient has ended by some lr a step.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "row_ops.cuh"

namespace cai {

constexpr int kAdamThreads = 256;
constexpr int kAdamShare = 3;                        // CTAs of an SM
constexpr int kAdamVec = 8;                          // elements of a thread at a time
constexpr int kAdamChunk = kAdamThreads * kAdamVec;  // elements that CTAs share the tensors out by
constexpr long long kAdamRun = 1 << 30;              // elements of a loop with 32-bit places
constexpr int kAdamGroup = 400;  // tensors of a launch: their gradients' addresses are its parameters

struct AdamTensor {
  void *param, *m, *v;
  uint8_t *m_scale, *v_scale;
  __nv_bfloat16* copy;
  long long n;
  long long first;  // its first chunk, counted over all tensors
  float decay;
  int16_t bf16;     // param's type
  int16_t wide;     // all buffers lie on the boundaries of the vector loads
};

struct AdamParams {
  const AdamTensor* table;
  int place, count;      // tensors of this launch
  long long first, last; // their chunks
  double lr, log_b1, log_b2;
  float b1, c1, b2, c2, eps;
  float rate, inv_root;  // of `step`
  float one;             // 1
  int step;
  uint32_t seed;
  const float* grad_scale;
  const float* lr_step;
  const void* grads[kAdamGroup];
};

// A mixer of 32 bits that a published search found to be nearly without bias (C. Wellons,
// "Prospecting for Hash Functions", 2018).
__device__ __forceinline__ uint32_t adam_mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float power_of(int byte) {
  return byte == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte ? byte << 23 : 0x00400000);
}
__device__ __forceinline__ float e4m3_value(uint8_t code) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
}
// The biased power of a block whose largest magnitude has the bits `top`.
__device__ __forceinline__ int power_for(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int b = static_cast<int>(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 0 ? 0 : b;
}
// x under the biased power `byte`, rounded up where 16 bits of dither carry; `least`:
// what a number that is not 0 has at least.
__device__ __forceinline__ uint32_t e4m3_code(float x, int byte, uint32_t dither, uint32_t least) {
  const float y = __fmul_rn(fabsf(x), __uint_as_float(static_cast<uint32_t>(254 - (byte < 254 ? byte : 0)) << 23));
  // E4M3's exponent and mantissa are those of y 2^-120 in fp32, denormals too.
  uint32_t code = (__float_as_uint(__fmul_rn(y, 0x1p-120f)) + (dither << 4)) >> 20;
  if (byte == 255) return 0;
  if (x != 0.0f && code == 0) code = least;
  return code | (__float_as_uint(x) >> 24 & (code != 0 ? 0x80u : 0u));
}
// Whether m's share of its gradient, (1 - beta1) g, is below the smallest number under
// the biased power `byte`.
__device__ __forceinline__ bool e4m3_below(float share, int byte) {
  return __fmul_rn(fabsf(share), __uint_as_float(static_cast<uint32_t>(254 - byte) << 23)) < 0x1p-9f;
}

// Two sums, each rounded once.  The compiler makes one operation of a packed product
// and the packed sum that takes it, explicit roundings or not; a product by a 1 that
// it does not know stands between them.
__device__ __forceinline__ float2 add2(float2 a, float2 b, float one) {
  return __ffma2_rn(a, make_float2(one, one), b);
}

// Eight elements as they are in memory, read and written once.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* p) {
    asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p));
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
  }
};
template <>
struct Eight<__nv_bfloat16> {
  uint4 x;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = ld_stream(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void values(float (&v)[8]) const { Row<__nv_bfloat16>::unpack(x, v); }
};
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  asm volatile("st.global.L1::no_allocate.v8.f32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"f"(x[0]), "f"(x[1]), "f"(x[2]),
               "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "l"(p)
               : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), Row<__nv_bfloat16>::pack(x));
}
// E4M3 codes and their block's power.
struct EightCodes {
  uint2 c;
  uint8_t power;
  __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* scale) {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(c.x), "=r"(c.y) : "l"(p));
    uint32_t b;
    asm volatile("ld.global.u8 %0, [%1];" : "=r"(b) : "l"(scale));
    power = static_cast<uint8_t>(b);
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
    const float scale = power_of(power);
    const uint32_t w[4] = {c.x & 0xffffu, c.x >> 16, c.y & 0xffffu, c.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[i]), __NV_E4M3);
      const float2 f = __fmul2_rn(__half22float2(__half2(h)), make_float2(scale, scale));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
};

// A step's numbers, the same for every element of a tensor.
struct AdamStep {
  float b1, c1, b2, c2, eps;
  float rate, inv_root, keep;  // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), 1 - lr decay
  float one;
  float scale;                 // of the gradients
  bool scaled;
};

__device__ __forceinline__ float reciprocal(float x) {  // to 1 ulp; x is normal (eps is), or inf: 0
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// kN (even) elements; `root` is v's square root, before and after (kBits 8).
template <int kBits, int kN>
__device__ __forceinline__ void adam_update(const AdamStep& s, float (&p)[kN], const float (&grad)[kN],
                                            float (&m)[kN], float (&v)[kN], float (&root)[kN]) {
  const auto both = [](float x) { return make_float2(x, x); };
#pragma unroll
  for (int e = 0; e < kN; e += 2) {
    float2 g = make_float2(grad[e], grad[e + 1]);
    if (s.scaled) g = __fmul2_rn(g, both(s.scale));
    float2 v2 = make_float2(v[e], v[e + 1]);
    if (kBits == 8) {
      const float2 r = make_float2(root[e], root[e + 1]);
      v2 = __fmul2_rn(r, r);
    }
    const float2 m2 =
        add2(__fmul2_rn(make_float2(m[e], m[e + 1]), both(s.b1)), __fmul2_rn(g, both(s.c1)), s.one);
    v2 = add2(__fmul2_rn(v2, both(s.b2)), __fmul2_rn(__fmul2_rn(g, g), both(s.c2)), s.one);
    const float2 r = make_float2(__fsqrt_rn(v2.x), __fsqrt_rn(v2.y));
    const float2 d = add2(__fmul2_rn(r, both(s.inv_root)), both(s.eps), s.one);
    const float2 u = __fmul2_rn(m2, both(-s.rate));
    const float2 x = add2(__fmul2_rn(make_float2(p[e], p[e + 1]), both(s.keep)),
                                __fmul2_rn(u, make_float2(reciprocal(d.x), reciprocal(d.y))), s.one);
    p[e] = x.x;
    p[e + 1] = x.y;
    m[e] = m2.x;
    m[e + 1] = m2.y;
    v[e] = v2.x;
    v[e + 1] = v2.y;
    root[e] = r.x;
    root[e + 1] = r.y;
  }
}

__device__ __forceinline__ float magnitude(const float (&x)[8]) {  // NaN kept
  float t = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) t = max_nan(t, fabsf(x[e]));
  return t;
}

// The E4M3 codes of eight elements' m and root under their blocks' biased powers; k:
// the first one's hash before its mixing.  An m that is not 0 may have the code 0: see
// settled_m.  (Its sign is set under a comparison: nvcc 13.0.88 puts a sign that is
// always set together with a wrong byte of the fourth code.)
__device__ __forceinline__ void e4m3_codes8(const float (&m)[8], int bm, const float (&root)[8], int bv, uint32_t k,
                                            uint2& cm, uint2& cv) {
  const float dm = __uint_as_float(static_cast<uint32_t>(254 - (bm < 254 ? bm : 0)) << 23);
  const float dv = __uint_as_float(static_cast<uint32_t>(254 - (bv < 254 ? bv : 0)) << 23);
  uint32_t wm[2] = {0u, 0u}, wv[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t h = adam_mix(k + 0x9e3779b1u * e);
    // E4M3's exponent and mantissa are those of y 2^-120 in fp32, denormals too.
    const float2 y = __fmul2_rn(__fmul2_rn(make_float2(fabsf(m[e]), root[e]), make_float2(dm, dv)),
                                make_float2(0x1p-120f, 0x1p-120f));
    uint32_t c = (__float_as_uint(y.x) + (h << 16 >> 12)) >> 20;
    uint32_t d = (__float_as_uint(y.y) + (h >> 16 << 4)) >> 20;
    if (m[e] != 0.0f) c |= __float_as_uint(m[e]) >> 24 & 0x80u;
    if (root[e] != 0.0f) d = max(d, 1u);
    wm[e / 4] |= c << (8 * (e & 3));
    wv[e / 4] |= d << (8 * (e & 3));
  }
  cm = bm == 255 ? make_uint2(0u, 0u) : make_uint2(wm[0], wm[1]);
  cv = bv == 255 ? make_uint2(0u, 0u) : make_uint2(wv[0], wv[1]);
}

// The bytes of w that are 0 but for their highest bit: that bit of theirs.
__device__ __forceinline__ uint32_t no_code(uint32_t w) { return ~((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) & 0x80808080u; }

// One tensor's elements [from, to), from a multiple of the chunk, to its end or
// another.
template <int kBits>
struct AdamRun {
  AdamTensor a;
  const void* grad;
  bool grad_bf16;
  AdamStep s;
  uint32_t key;  // of the hash, place and step in it

  __device__ __forceinline__ uint32_t key_at(long long i) const { return adam_mix(key + static_cast<uint32_t>(i >> 32)); }

  template <typename P, typename G, int kState>
  struct Group {
    Eight<P> p;
    Eight<G> g;
    EightCodes m, v;
    __device__ __forceinline__ void load(const AdamTensor& a, const G* grad, uint32_t j) {
      p.load(static_cast<const P*>(a.param) + j);
      g.load(grad + j);
      m.load(static_cast<const uint8_t*>(a.m) + j, a.m_scale + (j >> 5));
      v.load(static_cast<const uint8_t*>(a.v) + j, a.v_scale + (j >> 5));
    }
  };
  template <typename P, typename G>
  struct Group<P, G, 32> {
    Eight<P> p;
    Eight<G> g;
    Eight<float> m, v;
    __device__ __forceinline__ void load(const AdamTensor& a, const G* grad, uint32_t j) {
      p.load(static_cast<const P*>(a.param) + j);
      g.load(grad + j);
      m.load(static_cast<const float*>(a.m) + j);
      v.load(static_cast<const float*>(a.v) + j);
    }
  };

  // Eight codes of m, with those of 0 of numbers that are not 0 (`none`: their bytes' highest
  // bits) made 1 where the number keeps one.  Rare, so what it needs is read again: the
  // gradients, and the roots' codes before the new ones are written.  (A tensor of which
  // half the gradients end at once, here and there, 67 M elements: 215 us a step, 270 for some
  // while their m end.)
  template <typename G>
  __device__ __noinline__ uint64_t settled_m(uint64_t codes, uint64_t none, int power, const G* grad,
                                             const uint8_t* root) const {
#pragma unroll 1
    for (; none != 0; none &= none - 1) {
      const int bit = __ffsll(static_cast<long long>(none)) - 1, e = bit >> 3;
      if (root[e] == 0 || !e4m3_below(__fmul_rn(gradient(grad, e), s.c1), power))
        codes |= 1ull << (bit - 7);
      else
        codes &= ~(1ull << bit);
    }
    return codes;
  }
  template <typename G>
  __device__ __forceinline__ float gradient(const G* grad, long long i) const {
    const float g = Row<G>::to_float(grad[i]);
    return s.scaled ? __fmul_rn(g, s.scale) : g;
  }

  // Eight elements to a thread, blocks of 32 to four lanes; with 8-bit states the
  // next eight are on their way meanwhile.  At most 2^30 elements.
  template <typename P, typename G>
  __device__ __forceinline__ void wide(long long from, uint32_t count) const {
    const int lane = threadIdx.x & 31;
    const AdamStep s = this->s;
    AdamTensor a = this->a;
    a.param = static_cast<P*>(a.param) + from;
    a.m = static_cast<char*>(a.m) + from * (kBits / 8);
    a.v = static_cast<char*>(a.v) + from * (kBits / 8);
    a.m_scale += from >> 5;
    a.v_scale += from >> 5;
    if (a.copy) a.copy += from;
    const G* grad = static_cast<const G*>(this->grad) + from;
    uint32_t j = threadIdx.x * kAdamVec;
    Group<P, G, kBits> now;
    if (kBits == 8 && j < count) now.load(a, grad, j);
#pragma unroll 1
    for (; j < count; j += kAdamChunk) {
      if (kBits == 32) now.load(a, grad, j);
      float p[8], g[8], m[8], v[8], root[8];
      now.p.values(p);
      now.g.values(g);
      now.m.values(m);
      now.v.values(kBits == 32 ? v : root);
      adam_update<kBits>(s, p, g, m, v, root);
      store8(static_cast<P*>(a.param) + j, p);
      if (a.copy) store8(a.copy + j, p);
      if (kBits == 32) {
        store8(static_cast<float*>(a.m) + j, m);
        store8(static_cast<float*>(a.v) + j, v);
      } else {
        if (j + kAdamChunk < count) now.load(a, grad, j + kAdamChunk);
        const unsigned quad = 0xfu << (lane & 28);
        float tm = magnitude(m), tv = magnitude(root);
#pragma unroll
        for (int o = 1; o <= 2; o *= 2) {
          tm = max_nan(tm, __shfl_xor_sync(quad, tm, o));
          tv = max_nan(tv, __shfl_xor_sync(quad, tv, o));
        }
        const int bm = power_for(__float_as_uint(tm)), bv = power_for(__float_as_uint(tv));
        const long long i = from + j;
        uint2 cm, cv;
        e4m3_codes8(m, bm, root, bv, key_at(i) + 0x9e3779b1u * static_cast<uint32_t>(i), cm, cv);
        uint32_t none[2] = {no_code(cm.x), no_code(cm.y)};
        if ((none[0] | none[1]) != 0u && bm != 255) {
          uint32_t some[2] = {0u, 0u};  // the m that are not 0
#pragma unroll
          for (int e = 0; e < 8; ++e) some[e / 4] |= m[e] != 0.0f ? 0x80u << (8 * (e & 3)) : 0u;
          none[0] &= some[0];
          none[1] &= some[1];
          if ((none[0] | none[1]) != 0u) {
            const uint64_t codes =
                settled_m(static_cast<uint64_t>(cm.y) << 32 | cm.x, static_cast<uint64_t>(none[1]) << 32 | none[0], bm,
                          grad + j, static_cast<const uint8_t*>(a.v) + j);
            cm = make_uint2(static_cast<uint32_t>(codes), static_cast<uint32_t>(codes >> 32));
          }
        }
        __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + j), cm);
        __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + j), cv);
        if ((lane & 3) == 0) {
          a.m_scale[j >> 5] = static_cast<uint8_t>(bm);
          a.v_scale[j >> 5] = static_cast<uint8_t>(bv);
        }
      }
    }
  }

  // One element to a lane, whatever the alignment, blocks of 32 to `warps` warps in
  // turn.
  __device__ __noinline__ void narrow(long long from, long long to, int warp, int warps) const {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (long long b = from + warp * 32; b < to; b += warps * 32) {
      const long long i = b + lane;
      const bool in = i < to;
      float p[2] = {}, g[2] = {}, m[2] = {}, v[2] = {}, root[2] = {};
      bool had_root = false;
      if (in) {
        g[0] = grad_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(grad)[i]) : static_cast<const float*>(grad)[i];
        p[0] = a.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(a.param)[i]) : static_cast<const float*>(a.param)[i];
        if (kBits == 32) {
          m[0] = static_cast<const float*>(a.m)[i];
          v[0] = static_cast<const float*>(a.v)[i];
        } else {
          m[0] = __fmul_rn(e4m3_value(static_cast<const uint8_t*>(a.m)[i]), power_of(a.m_scale[i >> 5]));
          root[0] = __fmul_rn(e4m3_value(static_cast<const uint8_t*>(a.v)[i]), power_of(a.v_scale[i >> 5]));
          had_root = static_cast<const uint8_t*>(a.v)[i] != 0;
        }
        adam_update<kBits>(s, p, g, m, v, root);
        if (a.bf16)
          static_cast<__nv_bfloat16*>(a.param)[i] = __float2bfloat16_rn(p[0]);
        else
          static_cast<float*>(a.param)[i] = p[0];
        if (a.copy) a.copy[i] = __float2bfloat16_rn(p[0]);
      }
      if (kBits == 32) {
        if (in) {
          static_cast<float*>(a.m)[i] = m[0];
          static_cast<float*>(a.v)[i] = v[0];
        }
      } else {
        __syncwarp();
        const uint32_t h = adam_mix(key_at(i) + 0x9e3779b1u * static_cast<uint32_t>(i));
        const int bm = power_for(__reduce_max_sync(0xffffffffu, __float_as_uint(m[0]) & 0x7fffffffu));
        const int bv = power_for(__reduce_max_sync(0xffffffffu, __float_as_uint(root[0]) & 0x7fffffffu));
        if (in) {
          const float share = __fmul_rn(s.scaled ? __fmul_rn(g[0], s.scale) : g[0], s.c1);
          const bool ends = bm != 255 && had_root && e4m3_below(share, bm);
          static_cast<uint8_t*>(a.m)[i] = static_cast<uint8_t>(e4m3_code(m[0], bm, h & 0xffffu, ends ? 0u : 1u));
          static_cast<uint8_t*>(a.v)[i] = static_cast<uint8_t>(e4m3_code(root[0], bv, h >> 16, 1u));
        }
        if (lane == 0) {
          a.m_scale[i >> 5] = static_cast<uint8_t>(bm);
          a.v_scale[i >> 5] = static_cast<uint8_t>(bv);
        }
      }
    }
  }
};

// 32-bit states: the bytes bound it, 200 bf16 tensors of 242 M elements 813 us, 96 % of the
// copy's rate.  8-bit states: 75 instructions an element (a hash of 9, a root of 10, two
// encodings of 14) and 24 warps an SM cover the loads in part: a head of 518 M float32
// parameters with bf16 gradients and copies 1430 us, 86 % of the copy's rate.  (80 registers
// hold it but for 56 to 60 bytes.)  The next eight elements asked for before the update and not
// before the encoding: 1484, as more registers spill; with 2.7 rounds of CTAs instead of
// one 1552.
//
// The tensors with parameters of type P: every CTA takes an equal run of all
// tensors' chunks, one after another.
template <int kBits, typename P, typename G>
__global__ void __launch_bounds__(kAdamThreads, kAdamShare) adamw_kernel(const __grid_constant__ AdamParams p) {
  const int tid = threadIdx.x;
  const long long chunks = p.last - p.first;
  long long c = p.first + chunks * blockIdx.x / gridDim.x;
  const long long end = p.first + chunks * (blockIdx.x + 1) / gridDim.x;
  // The last tensor that begins at or before c (tensors of no elements begin where
  // the next one does).
  int at = -1;
#pragma unroll 1
  for (int i = 0; i < p.count; i += kAdamThreads)
    at += __syncthreads_count(i + tid < p.count && p.table[p.place + i + tid].first <= c);
  double lr = p.lr;
  uint32_t step = static_cast<uint32_t>(p.step);
  float rate = p.rate, inv_root = p.inv_root;
  if (p.lr_step) {  // by one thread: there are few units for 64 bits
    __shared__ float told[2];
    lr = p.lr_step[0];
    const double t = p.lr_step[1];
    step = static_cast<uint32_t>(t);
    if (tid == 0) {
      told[0] = static_cast<float>(lr / -expm1(t * p.log_b1));
      told[1] = static_cast<float>(1.0 / sqrt(-expm1(t * p.log_b2)));
    }
    __syncthreads();
    rate = told[0];
    inv_root = told[1];
  }
  // The tensor in turn, in shared memory: registers are for its elements.
  __shared__ AdamRun<kBits> run;
  const uint32_t key = adam_mix(adam_mix(p.seed) + step);
#pragma unroll 1
  for (; c < end; ++at) {
    const AdamTensor* row = p.table + p.place + at;
    const long long first = row->first, n = row->n;
    const long long last = min(end, first + (n + kAdamChunk - 1) / kAdamChunk);
    if (c >= last) continue;  // no elements
    const long long from = (c - first) * kAdamChunk, to = min(n, (last - first) * kAdamChunk);
    c = last;
    if (!p.grads[at] || row->bf16 != (sizeof(P) == 2)) continue;
    __syncthreads();
    if (tid == 0) {
      run.a = *row;
      run.grad = p.grads[at];
      run.grad_bf16 = sizeof(G) == 2;
      run.s = AdamStep{p.b1, p.c1, p.b2, p.c2, p.eps, rate, inv_root,
                       static_cast<float>(1.0 - lr * static_cast<double>(row->decay)), p.one,
                       p.grad_scale ? p.grad_scale[0] : 1.0f, p.grad_scale != nullptr};
      run.key = adam_mix(key + static_cast<uint32_t>(p.place + at));
    }
    __syncthreads();
    long long whole = from;
    if (run.a.wide && reinterpret_cast<uintptr_t>(run.grad) % (8 * sizeof(G)) == 0) {
      whole = to & ~31ll;
#pragma unroll 1
      for (long long at = from; at < whole; at += kAdamRun)
        run.template wide<P, G>(at, static_cast<uint32_t>(min(kAdamRun, whole - at)));
    }
    if (whole < to) run.narrow(whole, to, tid >> 5, kAdamThreads / 32);
  }
}

}  // namespace cai
