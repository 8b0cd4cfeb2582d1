// Sampling tokens from rows of logits (cai_sample_rows) and recording a row's K
// largest logits (cai_top_rows).
//
// With x_i = (z_i - max z) log2(e) / T, a token's weight is 2^x_i in units of
// 2^-40, rounded to a whole number.  Weights add up in 64 bits, so every sum is
// exact whatever its order: the same row gives the same token for any cluster
// size, and comparisons with a share of the whole do not hang on rounding.  A
// token below 2^-41 of the likeliest has no weight.
#pragma once

#include <climits>

#include "row_ops.cuh"
#include "softmax.cuh"

namespace cai {

constexpr float kRowLog2e = kLog2e;
constexpr float kWeightUnit = 1099511627776.0f;  // 2^40
constexpr int kTopMax = 512;                     // K of cai_top_rows

struct SampleParams {
  const void* logits;
  long long ld;
  int M, V;
  const float* temperature;  // each [M] or null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* prob;
};

// Calls f(element of the row, value) for what the thread keeps of the slice.
// What a vector holds besides the slice comes too, as -inf.
template <typename T, typename F>
__device__ __forceinline__ void for_slice(const Slice<T>& s, F&& f) {
  for (int v = threadIdx.x; v < s.n_vec; v += blockDim.x) {
    float z[Row<T>::kVec];
    Row<T>::unpack(s.vec[v], z);
    const int i0 = s.index(v, 0);
#pragma unroll
    for (int e = 0; e < Row<T>::kVec; ++e) f(i0 + e, z[e]);
  }
}

// 2^x of a logit relative to the largest.  Subtraction and product are rounded
// one by one, as the definition says.
__device__ __forceinline__ float row_exp2(float z, float zmax, float scale) {
  return exp2f(__fmul_rn(__fsub_rn(z, zmax), scale));
}
__device__ __forceinline__ unsigned long long weight_of(float e) {
  return __float2ull_rn(__fmul_rn(e, kWeightUnit));
}

template <typename T>
__device__ __forceinline__ float load_row_max(RowCta& c, const Slice<T>& s, const T* row) {
  float m = __uint_as_float(0xff800000u);
  load_slice<T, 4>(s, row, [&](const uint4& v) {
    float z[Row<T>::kVec];
    Row<T>::unpack(v, z);
#pragma unroll
    for (int e = 0; e < Row<T>::kVec; ++e) m = max_nan(m, z[e]);
  });
  row_begun();
  return __uint_as_float(
      static_cast<uint32_t>(cluster_reduce(c, __float_as_uint(m), MaxNanOp())));
}

// Elements above a key, and of those with that key the ones up to an index.
struct Kept {
  uint32_t key;
  int last;
  __device__ __forceinline__ bool has(uint32_t k, int i) const {
    return k > key || (k == key && i <= last);
  }
};

template <typename T>
__global__ void __launch_bounds__(kRowMaxThreads)
    sample_rows_kernel(const __grid_constant__ SampleParams p, int ctas) {
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  row_begin();
  RowCta c{&sh, static_cast<int>(cluster_ctarank()), ctas, 0};
  const int r = blockIdx.x / ctas;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T> s = row_slice(row, p.V, c.rank, ctas, slice_smem);
  const float t = p.temperature ? p.temperature[r] : 1.0f;
  const bool greedy = !(t > 0.0f);
  const float zmax = load_row_max(c, s, row);  // every CTA's slice is in place after it
  const float inf = __uint_as_float(0x7f800000u);
  const bool valid = fabsf(zmax) < inf;

  if (!valid || greedy) {
    // The first of the largest logits; a row without a softmax has no probability.
    int first = INT_MAX;
    unsigned long long mass = 0;
    for_slice(s, [&](int i, float z) {
      if (z == zmax && i >= s.lo && i < s.hi) first = min(first, i);
      if (valid) mass += weight_of(row_exp2(z, zmax, kRowLog2e));
    });
    const unsigned long long ix =
        cluster_reduce(c, static_cast<unsigned long long>(first),
                       [](unsigned long long a, unsigned long long b) { return a < b ? a : b; });
    __syncthreads();
    const unsigned long long whole = cluster_reduce(c, mass, AddOp());
    if (c.rank == 0 && threadIdx.x == 0) {
      p.token[r] = ix < static_cast<unsigned long long>(p.V) ? static_cast<int>(ix) : 0;
      p.prob[r] = valid ? static_cast<float>(static_cast<double>(kWeightUnit) /
                                             static_cast<double>(whole))
                        : __uint_as_float(0x7fc00000u);
    }
  } else {
    const float scale = fminf(fmaxf(__fdiv_rn(kRowLog2e, t), 1e-38f), 3e38f);
    const float pmin = p.min_p ? fminf(p.min_p[r], 1.0f) : 0.0f;
    const int k = p.top_k ? p.top_k[r] : 0;
    const float share = p.top_p ? p.top_p[r] : 1.0f;
    const uint32_t top = key_of<T>(zmax);
    Kept kept{0u, INT_MAX};
    if (k > 0 && k < p.V) {
      const Cut cut = find_cut<false>(c, top, k, [&](auto&& f) {
        for_slice(s, [&](int i, float z) {
          if (i >= s.lo && i < s.hi) f(key_of<T>(z), 0ull);
        });
      });
      kept.key = cut.key;
      const uint32_t need = k - cut.above.count;  // of the elements with the cut's key
      if (need < cut.at.count) {
        const auto tie = [&](int i) -> unsigned long long {
          return key_of<T>(Row<T>::to_float(s.data[i - s.lo])) == cut.key;
        };
        unsigned long long n = 0;
        for (int i = s.lo + threadIdx.x; i < s.hi; i += blockDim.x) n += tie(i);
        __syncthreads();
        const unsigned long long* parts = cluster_exchange(c, cta_reduce(c, n, AddOp()));
        kept.last = tell_index(c, find_index(c, s, parts, need - 1, tie));
      }
    }
    const auto weight = [&](int i, float z) -> unsigned long long {
      if (!kept.has(key_of<T>(z), i)) return 0;
      const float e = row_exp2(z, zmax, scale);
      return e < pmin ? 0 : weight_of(e);
    };
    const auto weight_at = [&](int i) { return weight(i, Row<T>::to_float(s.data[i - s.lo])); };
    unsigned long long mass = 0;
    for_slice(s, [&](int i, float z) { mass += weight(i, z); });
    __syncthreads();
    const unsigned long long* parts = cluster_exchange(c, cta_reduce(c, mass, AddOp()));
    unsigned long long whole = 0;
    for (int q = 0; q < ctas; ++q) whole += parts[q];
    if (share < 1.0f) {
      unsigned long long target = static_cast<unsigned long long>(
          ceil(static_cast<double>(share) * static_cast<double>(whole)));
      if (target < 1) target = 1;
      if (target > whole) target = whole;
      const Cut cut = find_cut<true>(c, top, target, [&](auto&& f) {
        for_slice(s, [&](int i, float z) {
          const unsigned long long w = weight(i, z);
          if (w) f(key_of<T>(z), w);
        });
      });
      const unsigned long long each = cut.at.mass / cut.at.count;
      const unsigned long long need = (target - cut.above.mass + each - 1) / each;
      int last = INT_MAX;
      if (need < cut.at.count) {
        const auto tie = [&](int i) -> unsigned long long {
          return key_of<T>(Row<T>::to_float(s.data[i - s.lo])) == cut.key && weight_at(i) != 0;
        };
        unsigned long long n = 0;
        for (int i = s.lo + threadIdx.x; i < s.hi; i += blockDim.x) n += tie(i);
        __syncthreads();
        const unsigned long long* tied = cluster_exchange(c, cta_reduce(c, n, AddOp()));
        last = tell_index(c, find_index(c, s, tied, need - 1, tie));
      }
      if (cut.key == kept.key) last = min(last, kept.last);
      kept = Kept{cut.key, last};
      mass = 0;
      for_slice(s, [&](int i, float z) { mass += weight(i, z); });
      __syncthreads();
      parts = cluster_exchange(c, cta_reduce(c, mass, AddOp()));
      whole = 0;
      for (int q = 0; q < ctas; ++q) whole += parts[q];
    }
    const float u = p.u[r] > 0.0f ? fminf(p.u[r], 1.0f) : 0.0f;  // NaN: 0
    unsigned long long drawn =
        static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(whole));
    if (drawn > whole - 1) drawn = whole - 1;
    const int ix = find_index(c, s, parts, drawn, weight_at);
    if (ix >= 0) {
      p.token[r] = ix;
      p.prob[r] = static_cast<float>(static_cast<double>(weight_at(ix)) /
                                     static_cast<double>(whole));
    }
  }
  row_sync();  // no CTA leaves while a peer may still write into it
}

struct TopParams {
  const void* logits;
  long long ld;
  int M, V, K;
  float temperature;
  float* values;   // [M, K]
  int32_t* index;  // [M, K]
  float* lse;      // [M]
};

struct AddFloatOp {  // on the bits of floats, in a fixed order
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return __float_as_uint(__uint_as_float(static_cast<uint32_t>(a)) +
                           __uint_as_float(static_cast<uint32_t>(b)));
  }
};

// Sorts n (a power of two) 64-bit values in shared memory, rising.
__device__ __forceinline__ void cta_sort(unsigned long long* a, int n) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int q = threadIdx.x; q < n / 2; q += blockDim.x) {
        const int i = (q / j) * 2 * j + q % j;
        const unsigned long long x = a[i], y = a[i + j];
        if ((x > y) == ((i & k) == 0)) {
          a[i] = y;
          a[i + j] = x;
        }
      }
      __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(kRowMaxThreads)
    top_rows_kernel(const __grid_constant__ TopParams p, int ctas) {
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  __shared__ unsigned long long list[kTopMax];
  __shared__ uint32_t placed;
  row_begin();
  RowCta c{&sh, static_cast<int>(cluster_ctarank()), ctas, 0};
  const int r = blockIdx.x / ctas;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T> s = row_slice(row, p.V, c.rank, ctas, slice_smem);
  const float zmax = load_row_max(c, s, row);
  const float scale = __fdiv_rn(kRowLog2e, p.temperature);
  float sum = 0.0f;
  for_slice(s, [&](int, float z) { sum += exp2f((z - zmax) * scale); });
  __syncthreads();
  sum = __uint_as_float(
      static_cast<uint32_t>(cluster_reduce(c, __float_as_uint(sum), AddFloatOp())));
  if (threadIdx.x == 0) placed = 0;

  Kept kept{0u, INT_MAX};
  const Cut cut = find_cut<false>(c, 0xffffffffu >> (32 - Row<T>::kKeyBits), p.K, [&](auto&& f) {
    for_slice(s, [&](int i, float z) {
      if (i >= s.lo && i < s.hi) f(key_of<T>(z), 0ull);
    });
  });
  kept.key = cut.key;
  const uint32_t need = p.K - cut.above.count;
  if (need < cut.at.count) {
    const auto tie = [&](int i) -> unsigned long long {
      return key_of<T>(Row<T>::to_float(s.data[i - s.lo])) == cut.key;
    };
    unsigned long long n = 0;
    for (int i = s.lo + threadIdx.x; i < s.hi; i += blockDim.x) n += tie(i);
    __syncthreads();
    const unsigned long long* parts = cluster_exchange(c, cta_reduce(c, n, AddOp()));
    kept.last = tell_index(c, find_index(c, s, parts, need - 1, tie));
  }
  unsigned long long n = 0;
  for_slice(s, [&](int i, float z) {
    n += i >= s.lo && i < s.hi && kept.has(key_of<T>(z), i);
  });
  __syncthreads();
  const unsigned long long* parts = cluster_exchange(c, cta_reduce(c, n, AddOp()));
  uint32_t base = 0;
  for (int q = 0; q < c.rank; ++q) base += static_cast<uint32_t>(parts[q]);
  for_slice(s, [&](int i, float z) {
    const uint32_t key = key_of<T>(z);
    if (i >= s.lo && i < s.hi && kept.has(key, i)) {
      const uint32_t at = base + atomicAdd(&placed, 1u);
      if (at < kTopMax)
        st_peer(list + at, 0, (static_cast<unsigned long long>(~key) << 32) | static_cast<uint32_t>(i));
    }
  });
  row_sync();
  if (c.rank != 0) return;  // nothing is written into the other CTAs any more
  int size = 1;
  while (size < p.K) size <<= 1;
  for (int i = p.K + threadIdx.x; i < size; i += blockDim.x) list[i] = ~0ull;
  __syncthreads();
  cta_sort(list, size);
  for (int i = threadIdx.x; i < p.K; i += blockDim.x) {
    const unsigned long long x = list[i];
    const uint32_t key = ~static_cast<uint32_t>(x >> 32);
    p.values[static_cast<long long>(r) * p.K + i] = value_of_key<T>(key);
    p.index[static_cast<long long>(r) * p.K + i] = static_cast<int32_t>(static_cast<uint32_t>(x));
  }
  if (threadIdx.x == 0) {
    const float inf = __uint_as_float(0x7f800000u);
    p.lse[r] = fabsf(zmax) < inf ? __fdiv_rn(zmax, p.temperature) + logf(sum) : zmax;
  }
}

}  // namespace cai
