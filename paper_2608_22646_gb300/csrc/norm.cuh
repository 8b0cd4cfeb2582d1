// Layer norm and RMS norm of rows, and their gradients (cai_norm_rows,
// cai_norm_backward).
//   xh = (x - mean) rstd,  y = xh w + b,
//   gx = rstd (g - mean g - xh mean(g xh)) with g = gy w  (RMS: without mean g),
//   gw = sum over rows of gy xh,  gb = sum of gy.
// Bound by the rows' bytes: each is read once and stays in registers until it is
// written.  Where every row lies on 16-byte boundaries a thread takes vectors of 16
// bytes (kWide), else single elements.  Rows that start anywhere, but as far behind a
// boundary in all arrays, are taken as wide ones too (kEdges): every eighth row lies
// alike, whatever the stride, so that a CTA that takes only such rows has fixed columns in
// its items; those at a row's ends begin before it or end behind it, and what is not the
// row's is masked.
#pragma once

#include <type_traits>

#include "async_copy.cuh"
#include "row_ops.cuh"
#include "vector_parts.cuh"

namespace cai {

struct NormParams {
  const void* x;
  long long ld;
  const void* gy;
  long long ld_gy;
  int M, H;
  bool layer;
  const void* weight;  // [H] or null
  const void* bias;
  float eps;
  float* stats;        // [M, 2]: mean and rstd, or null
  void* out;           // y or gx
  long long ld_out;
  float* part;         // [parts, 2, H] partial sums of gw and gb
  int parts;
  void *gw, *gb;
};

constexpr int kNormMaxH = 16384;
constexpr int kNormSms = 152;  // the partial sums' number does not follow the device
constexpr int kNormRingThreads = 512;

// Values come in pairs, which the packed operations take, or one by one.
template <typename P>
__device__ __forceinline__ P splat(float x);
template <>
__device__ __forceinline__ float2 splat<float2>(float x) {
  return make_float2(x, x);
}
template <>
__device__ __forceinline__ float splat<float>(float x) {
  return x;
}
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float mul(float a, float b) { return a * b; }
__device__ __forceinline__ float fma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ void put(float* p, float2 a) {
  p[0] = a.x;
  p[1] = a.y;
}
__device__ __forceinline__ void put(float* p, float a) { *p = a; }
__device__ __forceinline__ float whole(float2 a) { return a.x + a.y; }
__device__ __forceinline__ float whole(float a) { return a; }

// What a thread loads and stores at once: kN elements as they are in memory.
template <typename T, bool kWide>
struct Item;
template <typename T>
struct Item<T, true> {
  using P = float2;
  static constexpr int kN = Row<T>::kVec, kPairs = kN / 2;
  uint4 v;
  __device__ __forceinline__ void load(const T* p) { v = ld_stream(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void values(float2 (&f)[kPairs]) const {
    float x[kN];
    Row<T>::unpack(v, x);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = make_float2(x[2 * e], x[2 * e + 1]);
  }
  __device__ __forceinline__ void clear() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ static uint4 packed(const float2 (&f)[kPairs]) {
    float x[kN];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      x[2 * e] = f[e].x;
      x[2 * e + 1] = f[e].y;
    }
    return Row<T>::pack(x);
  }
  __device__ __forceinline__ static void store(T* p, const float2 (&f)[kPairs]) {
    __stcs(reinterpret_cast<uint4*>(p), packed(f));
  }
  // Items of which columns [0, H) are a part; p and i are the first element's.
  __device__ __forceinline__ static bool in(int i, int e, int H) { return static_cast<unsigned>(i + e) < static_cast<unsigned>(H); }
  __device__ __forceinline__ void load_part(const T* p, int i, int H) {
    clear();
#pragma unroll
    for (int e = 0; e < kN; ++e)
      if (in(i, e, H)) reinterpret_cast<T*>(&v)[e] = p[e];
  }
  __device__ __forceinline__ void keep_part(const uint4& bits) {
    v = make_uint4(v.x & bits.x, v.y & bits.y, v.z & bits.z, v.w & bits.w);
  }
  __device__ __forceinline__ static void store_part(T* p, const float2 (&f)[kPairs], int i, int H) {
    if (i < 0)
      store_from(p, packed(f), -i);
    else
      store_front(p, packed(f), H - i);
  }
};
template <typename T>
struct Item<T, false> {
  using P = float;
  static constexpr int kN = 1, kPairs = 1;
  float v;
  __device__ __forceinline__ void load(const T* p) { v = Row<T>::to_float(*p); }
  __device__ __forceinline__ void values(float (&f)[1]) const { f[0] = v; }
  __device__ __forceinline__ void clear() { v = 0.0f; }
  __device__ __forceinline__ static void store(T* p, const float (&f)[1]) { *p = Row<T>::from_float(f[0]); }
};

// kN elements of a weight (or bias), `none` where there is none; through L1, which
// keeps it.  `wide`: it lies on 32-byte boundaries.
template <typename W>
__device__ __forceinline__ void vector_values(const void* w, bool, int i, float none, float (&f)[1]) {
  f[0] = w ? Row<W>::to_float(static_cast<const W*>(w)[i]) : none;
}
template <typename W>
__device__ __forceinline__ void vector_values(const void* w, bool wide, int i, float none, float2 (&f)[2]) {
  const W* p = static_cast<const W*>(w) + i;
  if (!w) {
    f[0] = f[1] = splat<float2>(none);
  } else if (wide && sizeof(W) == 4) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p));
    f[0] = make_float2(v.x, v.y);
    f[1] = make_float2(v.z, v.w);
  } else {
    f[0] = make_float2(Row<W>::to_float(p[0]), Row<W>::to_float(p[1]));
    f[1] = make_float2(Row<W>::to_float(p[2]), Row<W>::to_float(p[3]));
  }
}
template <typename W>
__device__ __forceinline__ void vector_values(const void* w, bool wide, int i, float none, float2 (&f)[4]) {
  const W* p = static_cast<const W*>(w) + i;
  if (!w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = splat<float2>(none);
  } else if (wide && sizeof(W) == 4) {  // (two loads of 16 bytes would go over the lines twice)
    asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(f[0].x), "=f"(f[0].y), "=f"(f[1].x), "=f"(f[1].y), "=f"(f[2].x), "=f"(f[2].y), "=f"(f[3].x),
                   "=f"(f[3].y)
                 : "l"(p));
  } else if (wide) {
    float x[8];
    Row<__nv_bfloat16>::unpack(__ldg(reinterpret_cast<const uint4*>(p)), x);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = make_float2(x[2 * e], x[2 * e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = make_float2(Row<W>::to_float(p[2 * e]), Row<W>::to_float(p[2 * e + 1]));
  }
}
__device__ __forceinline__ bool wide_vector(const void* w) { return reinterpret_cast<uintptr_t>(w) % 32 == 0; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

constexpr int kNormMaxWarps = 16;

// Elements from the 16-byte boundary in front of a row to it.
template <typename T>
__device__ __forceinline__ int row_phase(const T* row) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
}

// The elements from i on that are in [0, H), 0 beside them.
template <typename W, int kPairs>
__device__ __forceinline__ void vector_part(const void* w, int i, int H, float none, float2 (&f)[kPairs]) {
  const auto one = [&](int c) {
    return c < 0 || c >= H ? 0.0f : w ? Row<W>::to_float(static_cast<const W*>(w)[c]) : none;
  };
#pragma unroll
  for (int e = 0; e < kPairs; ++e) f[e] = make_float2(one(i + 2 * e), one(i + 2 * e + 1));
}

// Of a thread's items, the first from column `lowest` on: the one that column H cuts, or -1.
template <int kN, int kItems>
__device__ __forceinline__ int tail_item(int lowest, int H) {
  const int k = (H - 1 - lowest) / (32 * kN), i = lowest + k * 32 * kN;
  return lowest < H && k < kItems && i < H && i + kN > H ? k : -1;
}

// Which elements of a row's first and of its last item are the row's: their bits, and 1
// and 0.  A CTA's rows lie alike, so they share it.
template <typename T>
struct RowEnds {
  static constexpr int kN = 16 / sizeof(T);
  uint4 bits[2];
  float ones[2][8];
  __device__ __forceinline__ void set(int tid, int phase, int H) {  // by 2 kN threads
    if (tid >= 2 * kN) return;
    const int e = tid % kN, end = (H + phase) % kN;
    const bool in = tid < kN ? e >= phase : end == 0 || e < end;
    ones[tid / kN][e] = in ? 1.0f : 0.0f;
    reinterpret_cast<std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>*>(&bits[tid / kN])[e] = in ? ~0u : 0u;
  }
  // Values of the first or the last item made 0 outside the row.
  __device__ __forceinline__ void keep(float2* f, int last) const {
    const float4* m = reinterpret_cast<const float4*>(ones[last]);
#pragma unroll
    for (int k = 0; k < kN / 4; ++k) {
      const float4 q = m[k];
      f[2 * k] = mul(f[2 * k], make_float2(q.x, q.y));
      f[2 * k + 1] = mul(f[2 * k + 1], make_float2(q.z, q.w));
    }
  }
};


// Weight and bias as floats in shared memory: [2, H], 4 of each item's elements
// together, so that a warp's loads of 16 bytes lie side by side.
__host__ __device__ inline int staged_cols(int n) { return (n + 7) & ~7; }
template <int kN>
__device__ __forceinline__ int staged_at(int i, int H) {
  return kN == 8 ? (i >> 2 & 1) * (H / 2) + (i >> 3) * 4 + (i & 3) : i;
}
__device__ __forceinline__ void staged_values(const float* v, int H, int i, float2 (&f)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(v + i / 2);
  const float4 b = *reinterpret_cast<const float4*>(v + H / 2 + i / 2);
  f[0] = make_float2(a.x, a.y);
  f[1] = make_float2(a.z, a.w);
  f[2] = make_float2(b.x, b.y);
  f[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ void staged_values(const float* v, int, int i, float2 (&f)[2]) {
  const float4 a = *reinterpret_cast<const float4*>(v + i);
  f[0] = make_float2(a.x, a.y);
  f[1] = make_float2(a.z, a.w);
}
__device__ __forceinline__ void staged_values(const float* v, int, int i, float (&f)[1]) { f[0] = v[i]; }

// A row to `warps` warps, kItems items to a thread; a CTA of more warps has several such
// groups, each with a barrier of its own.  Mean and variance one after the other from
// registers.  kStage: weight and bias once into shared memory, for CTAs that take many
// rows; from L1 every row's would cost more than the row (16384 rows of 4096 bf16,
// float32 weight and bias: 54 us, L1 busy for 77 % of them; two rows at a time that
// share them 66; staged, with the next row on its way, 49; the rows' bytes take 39.6).
// kEdges: 16000 rows of 4099 bf16 75 us (an element at a time 277; through a ring as below,
// whose masks spill, 125), 30000 of 1025 48 (150).
template <typename T, typename W, bool kWide, int kItems, bool kStage, bool kEdges = false>
__global__ void __launch_bounds__(512, kItems * Item<T, kWide>::kN * sizeof(T) > 128 ? 1 : 2)
    norm_rows_kernel(const __grid_constant__ NormParams p, int warps) {
  using It = Item<T, kWide>;
  using P = typename It::P;
  constexpr int kN = It::kN, kPairs = It::kPairs;
  extern __shared__ __align__(16) float staged[];
  __shared__ float red[4][kNormMaxWarps];
  const bool wide_w = wide_vector(p.weight), wide_b = wide_vector(p.bias);
  const int span = warps * 32, groups = blockDim.x / span, group = threadIdx.x / span;
  const int at = threadIdx.x % span, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first_warp = group * warps;
  // Rows that groups take; a CTA's lie alike.  kEdges: `phase` elements behind a 16-byte
  // boundary, x and y alike, so that items begin before a row and end behind it.
  const long long step = static_cast<long long>(gridDim.x) * groups;
  const long long row0 = kStage ? static_cast<long long>(group) * gridDim.x + blockIdx.x
                                : static_cast<long long>(blockIdx.x) * groups + group;
  const int phase = kEdges ? row_phase(static_cast<const T*>(p.x) + blockIdx.x * p.ld) : 0, lowest = at / 32 * (32 * kN * kItems) + lane * kN - phase;
  const int cols = kEdges ? staged_cols(p.H + phase) : p.H;
  const auto col = [&](int k) { return lowest + k * 32 * kN; };
  const bool head = kEdges && lowest < 0;  // item 0 begins before the row
  const int tail = kEdges ? tail_item<kN, kItems>(lowest, p.H) : -1;  // the item that ends behind it, or -1
  const auto edge = [&](int k) { return kEdges && ((k == 0 && head) || k == tail); };
  __shared__ __align__(16) RowEnds<T> ends;
  if (kEdges) ends.set(threadIdx.x, phase, p.H);
  if (kStage) {
#pragma unroll 4
    for (int i = threadIdx.x; i < cols; i += blockDim.x) {
      const int c = i - phase;
      const bool in = c >= 0 && c < p.H;
      staged[staged_at<kN>(i, cols)] = in && p.weight ? Row<W>::to_float(static_cast<const W*>(p.weight)[c]) : 1.0f;
      staged[cols + staged_at<kN>(i, cols)] = in && p.bias ? Row<W>::to_float(static_cast<const W*>(p.bias)[c]) : 0.0f;
    }
    __syncthreads();
  }
  int turn = 0;
  const auto row_sum = [&](float v) {
    v = warp_sum(v);
    if (warps == 1) return v;
    float* slot = red[turn++ & 3];  // (written again after three more barriers)
    if (lane == 0) slot[warp] = v;
    if (kStage)
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(span) : "memory");
    else
      __syncthreads();  // (a CTA of one row)
    v = slot[first_warp];
#pragma unroll 1
    for (int i = 1; i < warps; ++i) v += slot[first_warp + i];
    return v;
  };
  const auto load = [&](It(&it)[kItems], long long r) {
    const T* x = static_cast<const T*>(p.x) + r * p.ld + lowest;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = col(k);
      if constexpr (kEdges) {
        if ((r == 0 && i < 0) || (r == p.M - 1 && i < p.H && i + kN > p.H)) {
          it[k].load_part(x + k * 32 * kN, i, p.H);  // the rest is in front of or behind all rows
          continue;
        }
      }
      if (i < p.H) it[k].load(x + k * 32 * kN); else it[k].clear();
    }
  };
  It it[kItems], next[kStage ? kItems : 1];  // kStage: the next row is on its way meanwhile
  if constexpr (kStage)
    if (row0 < p.M) load(next, row0);
#pragma unroll 1
  for (long long r = row0; r < p.M; r += step) {
    if constexpr (kStage) {
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        it[k] = next[k];
        if constexpr (kEdges)
          if (edge(k)) it[k].keep_part(ends.bits[k == tail]);
      }
      if (r + step < p.M) load(next, r + step);
    } else {
      load(it, r);
    }
    float mean = 0.0f;
    if (p.layer) {
      P sum = splat<P>(0.0f);
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        P f[kPairs];
        it[k].values(f);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) sum = add(sum, f[e]);
      }
      mean = __fdiv_rn(row_sum(whole(sum)), p.H);
    }
    const P off = splat<P>(-mean);
    P sum = splat<P>(0.0f);
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      if (col(k) < p.H) {
        P f[kPairs];
        it[k].values(f);
        if constexpr (kEdges) {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) f[e] = add(f[e], off);
          if (edge(k)) ends.keep(f, k == tail);
#pragma unroll
          for (int e = 0; e < kPairs; ++e) sum = fma(f[e], f[e], sum);
        } else {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            const P d = add(f[e], off);
            sum = fma(d, d, sum);
          }
        }
      }
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(row_sum(whole(sum)), p.H) + p.eps));
    T* y = static_cast<T*>(p.out) + r * p.ld_out + lowest;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = col(k);
      if (i < p.H) {
        P f[kPairs], w[kPairs], b[kPairs];
        it[k].values(f);
        if (kStage) {
          staged_values(staged, cols, i + phase, w);
          staged_values(staged + cols, cols, i + phase, b);
        } else {
          vector_values<W>(p.weight, wide_w, i, 1.0f, w);
          vector_values<W>(p.bias, wide_b, i, 0.0f, b);
        }
#pragma unroll
        for (int e = 0; e < kPairs; ++e) f[e] = fma(mul(add(f[e], off), splat<P>(rstd)), w[e], b[e]);
        if constexpr (kEdges) {
          if (edge(k)) {
            It::store_part(y + k * 32 * kN, f, i, p.H);
            continue;
          }
        }
        It::store(y + k * 32 * kN, f);
      }
    }
    if (at == 0 && p.stats) {
      p.stats[2 * r] = mean;
      p.stats[2 * r + 1] = rstd;
    }
  }
}

// Many wide rows on 16-byte boundaries: they come by asynchronous copies of 16 bytes through
// a ring in shared memory, each into a place that its own thread reads.  A CTA to an SM; its
// units of `span` threads take rows in turn, with a barrier each.  Weight and bias of a
// thread's columns stay in registers, which the kernel above leaves to rows.  bf16, 32
// elements to a thread: 16384 rows of 5120 63 us (88 above), 4096 of 16384 58 (86), of 49.4 and
// 39.5; 16384 of 4096 the same.  float32, 16 elements: 6500 rows of 5120 49 us (68; 32 elements
// 55).
template <typename T, typename W, int kElems, int kThreads>
__global__ void __launch_bounds__(kThreads, 1)
    norm_ring_kernel(const __grid_constant__ NormParams p, int span, int ring) {
  using It = Item<T, true>;
  using P = float2;
  constexpr int kN = It::kN, kItems = kElems / kN, kPairs = It::kPairs, kCols = kItems * kPairs;
  extern __shared__ __align__(16) unsigned char norm_smem[];
  __shared__ __align__(16) float red[4][4 * kNormMaxWarps];
  const int nt = blockDim.x, units = nt / span, lane = threadIdx.x & 31, warps = span / 32;
  const int at = threadIdx.x % span, unit = threadIdx.x / span, warp = at / 32;
  const int slots = (warps + 3) & ~3, first = unit * slots;
  const long long step = static_cast<long long>(gridDim.x) * units;
  const int lowest = at / 32 * (32 * kElems) + lane * kN;
  const auto col = [&](int k) { return lowest + k * 32 * kN; };
  const long long row0 = static_cast<long long>(unit) * gridDim.x + blockIdx.x;
  constexpr int row_items = kItems * kThreads;
  It* const places = reinterpret_cast<It*>(norm_smem) + threadIdx.x;  // item k at [k kThreads]
  long long ask_row = row0;
  int ask_place = 0;
  const auto ask = [&]() {
    if (ask_row < p.M) {
      const T* x = static_cast<const T*>(p.x) + ask_row * p.ld + lowest;
      It* to = places + ask_place;
#pragma unroll
      for (int k = 0; k < kItems; ++k)
        if (col(k) < p.H) copy_async16(to + k * kThreads, x + k * 32 * kN);
    }
    copy_commit();
    ask_row += step;
    ask_place += row_items;
    if (ask_place == ring * row_items) ask_place = 0;
  };
  // (columns past the row's end are never copied: 0)
  for (int k = 0; k < ring * kItems; ++k) places[k * kThreads].clear();
  for (int k = 0; k < ring; ++k) ask();
  if (at < 16) red[at >> 2][first + slots - 4 + (at & 3)] = 0.0f;
  const bool wide_w = wide_vector(p.weight), wide_b = wide_vector(p.bias);
  P w[kCols], b[kCols];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int i = col(k);
    P f[kPairs], g[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = g[e] = splat<P>(0.0f);
    if (i < p.H) {
      vector_values<W>(p.weight, wide_w, i, 1.0f, f);
      vector_values<W>(p.bias, wide_b, i, 0.0f, g);
    }
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      w[k * kPairs + e] = f[e];
      b[k * kPairs + e] = g[e];
    }
  }
  __syncthreads();
  int turn = 0;
  const auto row_sum = [&](float v) {
    v = warp_sum(v);
    float* slot = red[turn++ & 3] + first;  // (written again after three more barriers)
    if (lane == 0) slot[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(unit + 1), "r"(span) : "memory");
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll 1
    for (int i = 0; i < warps; i += 4) {
      const float4 q = *reinterpret_cast<const float4*>(slot + i);
      sum = __fadd2_rn(sum, __fadd2_rn(make_float2(q.x, q.y), make_float2(q.z, q.w)));
    }
    return sum.x + sum.y;
  };
  int place = 0;
#pragma unroll 1
  for (long long r = row0; r < p.M; r += step) {
    copy_wait(ring - 1);
    const It* row = places + place;
    place += row_items;
    if (place == ring * row_items) place = 0;
    P x[kCols];
    P sum = splat<P>(0.0f);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      P f[kPairs];
      row[k * kThreads].values(f);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        x[k * kPairs + e] = f[e];
        sum = add(sum, f[e]);
      }
    }
    ask();
    const float mean = p.layer ? __fdiv_rn(row_sum(whole(sum)), p.H) : 0.0f;
    const P off = splat<P>(-mean);
    sum = splat<P>(0.0f);
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      if (col(k) < p.H) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          P& d = x[k * kPairs + e];
          d = add(d, off);
          sum = fma(d, d, sum);
        }
      }
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(row_sum(whole(sum)), p.H) + p.eps));
    T* y = static_cast<T*>(p.out) + r * p.ld_out + lowest;
    const P scale = splat<P>(rstd);
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      if (col(k) < p.H) {
        P f[kPairs];
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          const int c = k * kPairs + e;
          f[e] = fma(mul(x[c], scale), w[c], b[c]);
        }
        It::store(y + k * 32 * kN, f);
      }
    if (at == 0 && p.stats) {
      p.stats[2 * r] = mean;
      p.stats[2 * r + 1] = rstd;
    }
  }
}

// The backward call's plan, from H and M and never from the device: elements of a thread
// and threads of a unit (of H alone), which takes rows in turn and adds up its own
// partial sums; and the parts that the workspace has room for, one to a row and at most
// norm_share to an SM.  Units of a warp share CTAs of eight.
struct NormPlan {
  int elems, threads, parts;
};
__host__ __device__ inline int norm_share(int threads) { return 512 / threads; }  // units, or CTAs, of an SM
__host__ __device__ inline NormPlan norm_plan(int M, int H) {
  const int elems = H <= 2048 ? 8 : H <= 8192 ? 16 : 32;
  const int threads = (H + elems * 32 - 1) / (elems * 32) * 32;
  const int most = kNormSms * norm_share(threads);
  return NormPlan{elems, threads, M < most ? M : most};
}

__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float4 plus(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// The sums over a unit of two values: half a warp adds up the one, half the other.  A
// slot of an odd number of warps has a 0 behind them.  (It is written again after the
// other's barrier, which all have passed with this one's values read.)
template <bool kGroups>
__device__ __forceinline__ float2 unit_sums(float one, float two, int warps, int warp, int lane, float2* slot,
                                            int group) {
  const bool low = lane < 16;
  __syncwarp();
  float half = (low ? one : two) + __shfl_xor_sync(0xffffffffu, low ? two : one, 16);
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) half += __shfl_xor_sync(0xffffffffu, half, o);
  if (warps == 1) return make_float2(__shfl_sync(0xffffffffu, half, 0), __shfl_sync(0xffffffffu, half, 16));
  if ((lane & 15) == 0) reinterpret_cast<float*>(slot + warp)[lane >> 4] = half;
  if (kGroups)
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
  else
    __syncthreads();
  float2 sums = make_float2(0.0f, 0.0f);
#pragma unroll 4
  for (int i = 0; i < warps; i += 2) {
    const float4 q = *reinterpret_cast<const float4*>(slot + i);
    sums = __fadd2_rn(sums, __fadd2_rn(make_float2(q.x, q.y), make_float2(q.z, q.w)));
  }
  return sums;
}

// All gradients in one pass over the rows: fewer rows than SMs, rows that lie anywhere, and
// rows of which shared memory has no room for two.  A thread keeps its columns' sums and the weight in registers (kElems 32:
// the weight in L1, and 280 to 336 bytes spill, of single elements 950 to 1020) and, where
// there is room, the next row on its way.
template <typename T, typename W, bool kWide, int kElems>
__global__ void __launch_bounds__(512, 1)
    norm_grad_kernel(const __grid_constant__ NormParams p, int span) {
  using It = Item<T, kWide>;
  using P = typename It::P;
  constexpr int kN = It::kN, kItems = kElems / kN, kPairs = It::kPairs;
  constexpr int kCols = kItems * kPairs;  // pairs of a thread's columns
  constexpr bool kAhead = 2 * kItems * sizeof(It) <= 64;
  __shared__ __align__(16) float2 red[2][kNormMaxWarps];
  const bool wide_w = wide_vector(p.weight);
  const int groups = blockDim.x / span, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = span / 32;
  const int at = threadIdx.x % span;
  const int unit = blockIdx.x * groups + threadIdx.x / span;
  const long long step = static_cast<long long>(gridDim.x) * groups;
  constexpr bool kKeepW = kElems <= 16;  // else from L1 each time
  P w[kKeepW ? kCols : 1], gw[kCols], gb[kCols];
  const auto weight = [&](int k, P(&f)[kPairs]) {
    const int i = (at + k * span) * kN;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = splat<P>(0.0f);
    if (i < p.H) vector_values<W>(p.weight, wide_w, i, 1.0f, f);
  };
  const auto kept = [&](int k, P(&f)[kPairs]) {
    if (!kKeepW) weight(k, f);
#pragma unroll
    for (int e = 0; e < kPairs; ++e)
      if (kKeepW) f[e] = w[kKeepW ? k * kPairs + e : 0];
  };
  It x_next[kItems], gy_next[kItems], x_now[kItems], gy_now[kItems];
  const auto load = [&](It(&xs)[kItems], It(&gys)[kItems], long long r) {
    const T* x = static_cast<const T*>(p.x) + r * p.ld;
    const T* gy = static_cast<const T*>(p.gy) + r * p.ld_gy;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = (at + k * span) * kN;
      if (i < p.H) {
        xs[k].load(x + i);
        gys[k].load(gy + i);
      } else {
        xs[k].clear();
        gys[k].clear();
      }
    }
  };
  if (kAhead && unit < p.M) load(x_next, gy_next, unit);
  if (warps > 1 && warps % 2 && threadIdx.x < 2) red[threadIdx.x][warps] = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    P f[kPairs];
    if (kKeepW) weight(k, f);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      if (kKeepW) w[kKeepW ? k * kPairs + e : 0] = f[e];
      gw[k * kPairs + e] = gb[k * kPairs + e] = splat<P>(0.0f);
    }
  }
  // (A CTA of one unit has the same rows in all its warps; units of a warp have no
  // barriers.)
  float2 stats_next = make_float2(0.0f, 0.0f);
  const auto stats_of = [&](long long r) { return make_float2(p.stats[2 * r], p.stats[2 * r + 1]); };
  if (unit < p.M) stats_next = stats_of(unit);
#pragma unroll 1
  for (long long r = unit, turn = 0; r < p.M; r += step, ++turn) {
    const float mean = p.layer ? stats_next.x : 0.0f, rstd = stats_next.y;
    if (r + step < p.M) stats_next = stats_of(r + step);
    if (kAhead) {
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        x_now[k] = x_next[k];
        gy_now[k] = gy_next[k];
      }
      if (r + step < p.M) load(x_next, gy_next, r + step);
    } else {
      load(x_now, gy_now, r);
    }
    const P off = splat<P>(-mean), scale = splat<P>(rstd);
    P flat = splat<P>(0.0f), along = splat<P>(0.0f);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      P x[kPairs], gy[kPairs], f[kPairs];
      x_now[k].values(x);
      gy_now[k].values(gy);
      kept(k, f);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const int c = k * kPairs + e;
        const P xh = mul(add(x[e], off), scale), g = mul(gy[e], f[e]);
        flat = add(flat, g);
        along = fma(g, xh, along);
        gw[c] = fma(gy[e], xh, gw[c]);
        gb[c] = add(gb[c], gy[e]);
      }
    }
    if (p.out) {
      const float2 sums = unit_sums<false>(whole(flat), whole(along), warps, warp, lane, red[turn & 1], 0);
      T* out = static_cast<T*>(p.out) + r * p.ld_out;
      // gx = g rstd - (flat + xh along) rstd
      const P down = splat<P>(p.layer ? -__fdiv_rn(sums.x, p.H) * rstd : 0.0f);
      const P by = splat<P>(-__fdiv_rn(sums.y, p.H) * rstd);
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int i = (at + k * span) * kN;
        if (i < p.H) {
          P x[kPairs], gy[kPairs], f[kPairs];
          x_now[k].values(x);
          gy_now[k].values(gy);
          kept(k, f);
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            const P xh = mul(add(x[e], off), scale);
            x[e] = fma(mul(gy[e], f[e]), scale, fma(xh, by, down));
          }
          It::store(out + i, x);
        }
      }
    }
  }
  if (!p.part) return;
  grid_launch_dependents();  // the sums' kernel
  if (unit >= p.parts) return;
  float* part = p.part + static_cast<size_t>(unit) * 2 * p.H;
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int i = (at + k * span) * kN;
    if (i < p.H) {
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        put(part + i + e * (kN / kPairs), gw[k * kPairs + e]);
        put(part + p.H + i + e * (kN / kPairs), gb[k * kPairs + e]);
      }
    }
  }
}

// The same for other rows: they come by asynchronous copies of 16
// bytes through a ring in shared memory, each into a place that its own thread reads,
// and what the second pass needs of a row stays in registers, so that its place is free
// before the row's sums are there (kElems 32, for wide rows: it is read again, and the
// weight is in shared memory).  One CTA to an SM, whose units, with a barrier each, add
// up their sums before they leave them: 152 parts instead of 304 at two units an SM.
// 16384 rows of 4096 bf16: 74 us, of 59.3 at the copy's rate, 6 of it the parts (rows
// from registers, a row ahead: 85; a CTA to a unit: 85; eight elements to a thread,
// 100); 65536 of 1024: 73 (101), 32768 of 2048: 72 (104).  kEdges: 30000 of 1025 bf16 58 us (an
// element at a time 277), 16000 of 4099 97.  The bytes on their way, 192 KB an SM, cover
// memory; what is left is the time from a row's last load to its sums, with four warps
// a scheduler.
template <typename T, typename W, int kElems, bool kEdges>
__global__ void __launch_bounds__(kNormRingThreads, 1)
    norm_grad_ring_kernel(const __grid_constant__ NormParams p, int span, int ring) {
  using It = Item<T, true>;
  using P = float2;
  constexpr int kN = It::kN, kItems = kElems / kN, kPairs = It::kPairs, kCols = kItems * kPairs;
  constexpr bool kHold = kElems <= 16;
  extern __shared__ __align__(16) unsigned char norm_smem[];
  __shared__ __align__(16) float2 red[2][2 * kNormMaxWarps];
  const bool wide_w = wide_vector(p.weight);
  const int nt = blockDim.x, groups = nt / span, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = span / 32;
  const int at = threadIdx.x % span, group = threadIdx.x / span, first = group * ((warps + 1) & ~1);
  const int unit = group * gridDim.x + blockIdx.x;
  const long long step = static_cast<long long>(gridDim.x) * groups;
  const float inv_h = __fdiv_rn(1.0f, p.H);
  // The first column of item k; kEdges: rows start `phase` elements behind a 16-byte
  // boundary, all of a CTA's alike, as do x, gy and out.
  const int phase = kEdges ? row_phase(static_cast<const T*>(p.x) + blockIdx.x * p.ld) : 0, lowest = at / 32 * (32 * kElems) + lane * kN - phase;
  const auto col = [&](int k) { return lowest + k * 32 * kN; };
  const bool head = kEdges && lowest < 0;  // item 0 begins before the row
  const int tail = kEdges ? tail_item<kN, kItems>(lowest, p.H) : -1;  // the item that ends behind it, or -1
  const auto edge = [&](int k) { return kEdges && ((k == 0 && head) || k == tail); };
  __shared__ __align__(16) RowEnds<T> ends;
  if (kEdges) {
    ends.set(threadIdx.x, phase, p.H);
    __syncthreads();
  }
  constexpr int kApart = kNormRingThreads, row_items = 2 * kItems * kApart;
  It* const places = reinterpret_cast<It*>(norm_smem) + threadIdx.x;  // item k of x at [k kApart], of gy at [(kItems + k) kApart]
  long long ask_row = unit;
  int ask_place = 0;
  const auto ask = [&]() {
    if (ask_row < p.M) {
      const T* x = static_cast<const T*>(p.x) + ask_row * p.ld + lowest;
      const T* gy = static_cast<const T*>(p.gy) + ask_row * p.ld_gy + lowest;
      It* to = places + ask_place;
#pragma unroll
      for (int k = 0; k < kItems; ++k)
        if (col(k) < p.H) {
          if (kEdges && ((ask_row == 0 && col(k) < 0) || (ask_row == p.M - 1 && col(k) + kN > p.H))) {
            to[k * kApart].load_part(x + k * 32 * kN, col(k), p.H);  // the rest is in front of or behind all rows
            to[(kItems + k) * kApart].load_part(gy + k * 32 * kN, col(k), p.H);
          } else {
            copy_async16(to + k * kApart, x + k * 32 * kN);
            copy_async16(to + (kItems + k) * kApart, gy + k * 32 * kN);
          }
        }
    }
    copy_commit();
    ask_row += step;
    ask_place += row_items;
    if (ask_place == ring * row_items) ask_place = 0;
  };
  // (columns past the row's end are never copied: 0)
  for (int k = 0; k < ring * 2 * kItems; ++k) places[k * kApart].clear();
  for (int k = 0; k < ring; ++k) ask();
  if (warps % 2 && at < 2) red[at][first + warps] = make_float2(0.0f, 0.0f);
  float* const staged = reinterpret_cast<float*>(norm_smem + static_cast<size_t>(ring) * row_items * sizeof(It));
  const int cols = kEdges ? staged_cols(p.H + phase) : p.H;
  if (!kHold) {
#pragma unroll 4
    for (int i = threadIdx.x; i < cols; i += nt) {
      const int c = i - phase;
      float v = 0.0f;
      if (c >= 0 && c < p.H) v = p.weight ? Row<W>::to_float(static_cast<const W*>(p.weight)[c]) : 1.0f;
      staged[staged_at<kN>(i, cols)] = v;
    }
    __syncthreads();
  }
  P w[kHold ? kCols : 1], gw[kCols], gb[kCols];
  const auto weight = [&](int k, P(&f)[kPairs]) {
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = kHold ? w[kHold ? k * kPairs + e : 0] : splat<P>(0.0f);
    if (!kHold && col(k) < p.H) staged_values(staged, cols, col(k) + phase, f);
  };
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int i = col(k);
    P f[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = splat<P>(0.0f);
    if (kHold && edge(k))
      vector_part<W>(p.weight, i, p.H, 1.0f, f);
    else if (kHold && i < p.H)
      vector_values<W>(p.weight, wide_w && phase == 0, i, 1.0f, f);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      if (kHold) w[kHold ? k * kPairs + e : 0] = f[e];
      gw[k * kPairs + e] = gb[k * kPairs + e] = splat<P>(0.0f);
    }
  }
  float2 stats_next = make_float2(0.0f, 0.0f);
  const auto stats_of = [&](long long r) { return make_float2(p.stats[2 * r], p.stats[2 * r + 1]); };
  if (unit < p.M) stats_next = stats_of(unit);
  int place = 0;
#pragma unroll 1
  for (long long r = unit, turn = 0; r < p.M; r += step, ++turn) {
    const float mean = p.layer ? stats_next.x : 0.0f, rstd = stats_next.y;
    if (r + step < p.M) stats_next = stats_of(r + step);
    copy_wait(ring - 1);
    It* const row = places + place;
    place += row_items;
    if (place == ring * row_items) place = 0;
    if (head) {
      row[0].keep_part(ends.bits[0]);
      row[kItems * kApart].keep_part(ends.bits[0]);
    }
    if (tail >= 0) {
      row[tail * kApart].keep_part(ends.bits[1]);
      row[(kItems + tail) * kApart].keep_part(ends.bits[1]);
    }
    const P off = splat<P>(-mean), scale = splat<P>(rstd);
    P flat = splat<P>(0.0f), along = splat<P>(0.0f);
    P held_xh[kHold ? kCols : 1], held_g[kHold ? kCols : 1];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      P x[kPairs], gy[kPairs], f[kPairs];
      row[k * kApart].values(x);
      row[(kItems + k) * kApart].values(gy);
      weight(k, f);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const int c = k * kPairs + e;
        const P xh = mul(add(x[e], off), scale), g = mul(gy[e], f[e]);
        if (kHold) {
          held_xh[kHold ? c : 0] = xh;
          held_g[kHold ? c : 0] = g;
        }
        flat = add(flat, g);
        along = fma(g, xh, along);
        gw[c] = fma(gy[e], xh, gw[c]);
        gb[c] = add(gb[c], gy[e]);
      }
    }
    if (kHold) ask();
    if (p.out) {
      const float2 sums = unit_sums<true>(whole(flat), whole(along), warps, warp - group * warps, lane, red[turn & 1] + first, group);
      T* out = static_cast<T*>(p.out) + r * p.ld_out + lowest;
      // gx = g rstd - (flat + xh along) rstd
      const P down = splat<P>(p.layer ? -sums.x * inv_h * rstd : 0.0f);
      const P by = splat<P>(-sums.y * inv_h * rstd);
#pragma unroll
      for (int k = 0; k < kItems; ++k)
        if (col(k) < p.H) {
          P x[kPairs], gy[kPairs], f[kPairs];
          if (!kHold) {
            row[k * kApart].values(x);
            row[(kItems + k) * kApart].values(gy);
            weight(k, f);
          }
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            const int c = kHold ? k * kPairs + e : 0;
            const P xh = kHold ? held_xh[c] : mul(add(x[e], off), scale), g = kHold ? held_g[c] : mul(gy[e], f[e]);
            x[e] = fma(g, scale, fma(xh, by, down));
          }
          if (edge(k))
            It::store_part(out + k * 32 * kN, x, col(k), p.H);
          else
            It::store(out + k * 32 * kN, x);
        }
    }
    if (!kHold) ask();
  }
  if (!p.part) return;
  grid_launch_dependents();  // the sums' kernel
  // The units' sums of a CTA become one.
  float* part = p.part + static_cast<size_t>(blockIdx.x) * 2 * p.H;
  float* to = part;
  if (groups > 1) {
    copy_wait(0);
    __syncthreads();
    to = reinterpret_cast<float*>(norm_smem) + static_cast<size_t>(group) * 2 * p.H;
  }
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int i = col(k);
    if (i >= p.H) continue;
#pragma unroll
    for (int e = 0; e < kN; ++e)
      if (!kEdges || It::in(i, e, p.H)) {
        to[i + e] = e & 1 ? gw[k * kPairs + e / 2].y : gw[k * kPairs + e / 2].x;
        to[p.H + i + e] = e & 1 ? gb[k * kPairs + e / 2].y : gb[k * kPairs + e / 2].x;
      }
  }
  if (groups == 1) return;
  __syncthreads();
  using V = std::conditional_t<kEdges, float, float4>;
  const V* all = reinterpret_cast<const V*>(norm_smem);
  const int n = 2 * p.H * sizeof(float) / sizeof(V);
#pragma unroll 2
  for (int i = threadIdx.x; i < n; i += nt) {
    V sum = all[i];
#pragma unroll 4
    for (int g = 1; g < groups; ++g) sum = plus(sum, all[g * n + i]);
    reinterpret_cast<V*>(part)[i] = sum;
  }
}

// The partial sums added up: two columns to a lane, the parts over the CTA's warps.
constexpr int kNormSumWarps = 16;
template <typename W>
__global__ void __launch_bounds__(32 * kNormSumWarps) norm_weight_sum_kernel(const __grid_constant__ NormParams p) {
  constexpr int kFlight = 10;  // 152 parts at once
  __shared__ float2 sums[kNormSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int i = (blockIdx.x * 32 + lane) * 2;
  float2 sum = make_float2(0.0f, 0.0f);
  grid_dependency_wait();
#pragma unroll 1
  for (int k = warp; k < p.parts; k += kNormSumWarps * kFlight) {
    float2 v[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int part = k + j * kNormSumWarps;
      v[j] = make_float2(0.0f, 0.0f);
      if (part < p.parts && i < 2 * p.H)
        v[j] = __ldcs(reinterpret_cast<const float2*>(p.part + static_cast<size_t>(part) * 2 * p.H + i));
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) sum = __fadd2_rn(sum, v[j]);
  }
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || i >= 2 * p.H) return;
#pragma unroll
  for (int k = 1; k < kNormSumWarps; ++k) sum = __fadd2_rn(sum, sums[k][lane]);
  const auto write = [&](int c, float v) {
    void* out = c < p.H ? p.gw : p.gb;
    if (out) static_cast<W*>(out)[c < p.H ? c : c - p.H] = Row<W>::from_float(v);
  };
  write(i, sum.x);
  write(i + 1, sum.y);
}

}  // namespace cai
