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

// Sums of weights in 32-bit pieces, a few instructions an element: e + 1 rounds
// e to units of 2^-23 and holds them in the low bits, what that leaves is exact
// and goes the same way in units of 2^-40, rounded as weight_of does.  Up to 511
// elements a thread.
struct WeightSum {
  static constexpr uint32_t kOne = 0x3f800000u;    // 1.0f
  static constexpr uint32_t kMagic = 0x4b400000u;  // 1.5 * 2^23
  uint32_t high = 0, low = 0;
  __device__ __forceinline__ void add(float e0, float e1) {
    const float2 e = make_float2(e0, e1), one = make_float2(1.0f, 1.0f);
    const float2 h = __fadd2_rn(e, one);
    const float2 r = __fadd2_rn(e, __fadd2_rn(one, make_float2(-h.x, -h.y)));
    const float2 l = __ffma2_rn(r, make_float2(kWeightUnit, kWeightUnit),
                                make_float2(12582912.0f, 12582912.0f));
    high += __float_as_uint(h.x) + __float_as_uint(h.y);
    low += __float_as_uint(l.x) + __float_as_uint(l.y);
  }
  // After n elements.
  __device__ __forceinline__ unsigned long long sum(uint32_t n) const {
    const long long lo = static_cast<int32_t>(low - n * kMagic);
    return (static_cast<unsigned long long>(high - n * kOne) << 17) + lo;
  }
};

// 2^x of a pair of logits relative to the largest, bit for bit row_exp2 where a
// weight remains.
__device__ __forceinline__ float2 row_exp2_pair(float z0, float z1, float zmax, float scale) {
  const float2 x = __fmul2_rn(__fadd2_rn(make_float2(z0, z1), make_float2(-zmax, -zmax)),
                              make_float2(scale, scale));
  return make_float2(fast_exp2(x.x), fast_exp2(x.y));
}

// Elements above a key, and of those with that key the ones up to an index.
struct Kept {
  uint32_t key;
  int last;
  __device__ __forceinline__ bool has(uint32_t k, int i) const {
    return k > key || (k == key && i <= last);
  }
};

// Loads the slice and returns the thread's largest logit.
template <typename T>
__device__ __forceinline__ float load_row(const Slice<T>& s, const T* row) {
  float m = __uint_as_float(0xff800000u);
  load_slice<T, 4>(s, row, [&](const uint4& v) { m = vec_max(v, m, T()); });
  return m;
}

// The row's largest logit, and a key with at least `want` elements of the row at
// or above it (0: none is known): every CTA finds one for its part of them.
struct Floor {
  float zmax;
  uint32_t key;
  // No element with that key or above is below it.
  template <typename T>
  __device__ __forceinline__ float low() const {
    const float v = value_of_key<T>(key);
    return v == v ? v : __uint_as_float(0xff800000u);
  }
};
template <typename T>
__device__ __forceinline__ Floor row_floor(RowCta& c, float thread_max, int want) {
  const uint32_t mine = want > 0 ? local_floor<T>(thread_max, (want + c.ctas - 1) / c.ctas) : 0u;
  const unsigned long long v[2] = {cta_reduce(c, __float_as_uint(thread_max), MaxNanOp()), mine};
  const Parts parts = cluster_exchange(c, v);
  Floor f{__uint_as_float(static_cast<uint32_t>(parts.of(0)[0])), static_cast<uint32_t>(parts.of(1)[0])};
  for (int i = 1; i < c.ctas; ++i) {
    f.zmax = max_nan(f.zmax, __uint_as_float(static_cast<uint32_t>(parts.of(0)[i])));
    f.key = min(f.key, static_cast<uint32_t>(parts.of(1)[i]));
  }
  return f;
}

// Pushes the elements of a vector whose key is at least `floor` (value `low`);
// returns how many.
template <typename T>
__device__ __forceinline__ uint32_t push_vector(const RowCta& c, const Slice<T>& s, int v,
                                                const float (&z)[Row<T>::kVec], uint32_t floor) {
  uint32_t n = 0;
#pragma unroll
  for (int e = 0; e < Row<T>::kVec; ++e) {
    const int i = s.index(v, e);
    const uint32_t key = key_of<T>(z[e]);
    if (key >= floor && i >= s.lo && i < s.hi) {
      push_candidate(c, key, i);
      ++n;
    }
  }
  return n;
}

// In CTA 0, with the candidates listed: sorts them, keeps, draws.  `whole`: the
// weight of all tokens that min-p leaves, where top-k is off.
template <typename T>
__device__ void sample_candidates(const RowCta& c, const SampleParams& p, int r, int n, int k,
                                  float zmax, float scale, float pmin, float share, float u,
                                  unsigned long long whole) {
  unsigned long long* list = c.sh->list;
  const int tid = threadIdx.x, nt = blockDim.x;
  const auto weight = [&](uint32_t key) -> unsigned long long {
    const float e = row_exp2(value_of_key<T>(key), zmax, scale);
    return e < pmin ? 0 : weight_of(e);
  };
  cta_sort_any(list, n);
  if (k > 0) n = min(n, k);
  const int per = (n + nt - 1) / nt;
  const int a = min(n, tid * per), b = min(n, a + per);
  unsigned long long own = 0, all;
  for (int i = a; i < b; ++i) own += weight(candidate_key(list[i]));
  unsigned long long run = cta_scan(c, own, all);
  if (k > 0) whole = all;
  // How many of the front are kept: their running weight is below the target
  // before them.
  unsigned long long target = ~0ull;
  if (share < 1.0f) {
    target = static_cast<unsigned long long>(
        ceil(static_cast<double>(share) * static_cast<double>(whole)));
    if (target < 1) target = 1;
  }
  int kept = 0, end = 0;
  for (int i = a; i < b; ++i) {
    const unsigned long long w = weight(candidate_key(list[i]));
    const bool keep = w != 0 && run < target;
    if (keep) {
      ++kept;
      end = i + 1;
    }
    // From here on in index order, the key behind it; the others last.
    list[i] = keep ? (static_cast<unsigned long long>(candidate_index(list[i])) << 32) |
                         candidate_key(list[i])
                   : ~0ull;
    run += w;
  }
  n = static_cast<int>(cta_reduce(c, end, MaxOp(), 1));
  unsigned long long n_kept;
  cta_scan(c, kept, n_kept);
  cta_sort_any(list, n);
  n = static_cast<int>(n_kept);
  const int per2 = (n + nt - 1) / nt;
  const int a2 = min(n, tid * per2), b2 = min(n, a2 + per2);
  own = 0;
  for (int i = a2; i < b2; ++i) own += weight(static_cast<uint32_t>(list[i]));
  run = cta_scan(c, own, all);
  unsigned long long drawn =
      static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(all));
  if (drawn > all - 1) drawn = all - 1;
  if (drawn < run || drawn >= run + own) return;
  for (int i = a2; i < b2; ++i) {
    const unsigned long long w = weight(static_cast<uint32_t>(list[i]));
    run += w;
    if (drawn < run) {
      p.token[r] = static_cast<int32_t>(list[i] >> 32);
      p.prob[r] = static_cast<float>(static_cast<double>(w) / static_cast<double>(all));
      return;
    }
  }
}

// Candidates asked for where only the weight limits what is kept.
constexpr int kNucleusWant = 256;

template <typename T>
__global__ void __launch_bounds__(kRowMaxThreads)
    sample_rows_kernel(const __grid_constant__ SampleParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  row_begin();
  RowCta c{&sh, static_cast<int>(cluster_ctarank()), ctas, 0};
  const int r = blockIdx.x / ctas;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T> s = row_slice(row, p.V, c.rank, ctas, slice_smem);
  if (threadIdx.x == 0) sh.listed = 0;
  const float t = p.temperature ? p.temperature[r] : 1.0f;
  const bool greedy = !(t > 0.0f);
  const float scale = greedy ? kRowLog2e : fminf(fmaxf(__fdiv_rn(kRowLog2e, t), 1e-38f), 3e38f);
  const float pmin = p.min_p ? fminf(p.min_p[r], 1.0f) : 0.0f;
  int k = p.top_k ? p.top_k[r] : 0;
  if (k >= p.V || k < 0) k = 0;
  const float share = p.top_p ? p.top_p[r] : 1.0f;
  const float u = p.u[r] > 0.0f ? fminf(p.u[r], 1.0f) : 0.0f;  // NaN: 0
  // Tokens that decide the row, if a list can hold them.
  const int want = greedy ? 0 : k > 0 ? (k <= kListMax / 2 ? k : 0) : share < 1.0f || pmin > 0.0f ? kNucleusWant : 0;

  const float thread_max = load_row(s, row);
  row_begun();
  const Floor floor = row_floor<T>(c, thread_max, p.V <= kListMax ? 0 : want);
  const float zmax = floor.zmax;
  const float inf = __uint_as_float(0x7f800000u);

  if (!(fabsf(zmax) < inf) || greedy) {
    // The first of the largest logits; a row without a softmax has no probability.
    const bool valid = fabsf(zmax) < inf;
    int first = INT_MAX;
    WeightSum sum;
    uint32_t n = 0;
    for (int v = threadIdx.x; v < s.n_vec; v += blockDim.x, n += kVec) {
      float z[kVec];
      Row<T>::unpack(s.vec[v], z);
#pragma unroll
      for (int e = kVec - 1; e >= 0; --e)
        if (z[e] == zmax && s.index(v, e) >= s.lo && s.index(v, e) < s.hi) first = min(first, s.index(v, e));
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const float2 w = row_exp2_pair(z[e], z[e + 1], zmax, scale);
        sum.add(w.x, w.y);
      }
    }
    const unsigned long long ix =
        cta_reduce(c, static_cast<unsigned long long>(first),
                   [](unsigned long long a, unsigned long long b) { return a < b ? a : b; }, 1);
    const unsigned long long v[2] = {cta_reduce(c, sum.sum(n), AddOp()), ix};
    const Parts parts = cluster_exchange(c, v);
    if (c.rank == 0 && threadIdx.x == 0) {
      unsigned long long best = parts.of(1)[0];
      for (int q = 1; q < ctas; ++q) best = min(best, parts.of(1)[q]);
      p.token[r] = best < static_cast<unsigned long long>(p.V) ? static_cast<int>(best) : 0;
      p.prob[r] = valid ? static_cast<float>(static_cast<double>(kWeightUnit) /
                                             static_cast<double>(parts.sum(ctas, 0)))
                        : __uint_as_float(0x7fc00000u);
    }
    return;  // no CTA writes into another from here on
  }

  // One pass: the weight of every token that min-p leaves (not needed under
  // top-k), and the candidates.
  const bool listing = want > 0 && (p.V <= kListMax || floor.key > 0);
  const float low = floor.low<T>();
  WeightSum sum;
  uint32_t n = 0, pushed = 0;
  unsigned long long listed_mass = 0;
  if (k > 0) {
    if (listing)
      for (int v = threadIdx.x; v < s.n_vec; v += blockDim.x)
        if (!(vec_max(s.vec[v], -inf, T()) < low)) {
          float z[kVec];
          Row<T>::unpack(s.vec[v], z);
          pushed += push_vector(c, s, v, z, floor.key);
        }
  } else {
    for (int v = threadIdx.x; v < s.n_vec; v += blockDim.x, n += kVec) {
      float z[kVec];
      Row<T>::unpack(s.vec[v], z);
      bool any = false;
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        float2 w = row_exp2_pair(z[e], z[e + 1], zmax, scale);
        w.x = w.x < pmin ? 0.0f : w.x;
        w.y = w.y < pmin ? 0.0f : w.y;
        sum.add(w.x, w.y);
        any |= z[e] >= low || z[e + 1] >= low;
      }
      if (listing && any) {
        pushed += push_vector(c, s, v, z, floor.key);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (key_of<T>(z[e]) >= floor.key) {
            const float w = row_exp2(z[e], zmax, scale);
            listed_mass += w < pmin ? 0 : weight_of(w);
          }
      }
    }
  }
  const unsigned long long sums[3] = {sum.sum(n), listed_mass, pushed};
  Parts parts = exchange_sums(c, sums);
  unsigned long long whole = parts.sum(ctas, 0);
  const unsigned long long n_listed = parts.sum(ctas, 2);
  if (listing && n_listed <= kListMax) {
    // All that is kept is listed: the first k; or enough weight for the target;
    // or min-p's lowest.
    bool all = k > 0;
    if (!all && share < 1.0f)
      all = static_cast<double>(parts.sum(ctas, 1)) >= ceil(static_cast<double>(share) * static_cast<double>(whole));
    if (!all) all = parts.sum(ctas, 1) == whole;
    if (all) {
      if (c.rank == 0)
        sample_candidates<T>(c, p, r, static_cast<int>(n_listed), k, zmax, scale, pmin, share, u, whole);
      return;
    }
  }

  const uint32_t top = key_of<T>(zmax);
  Kept kept{0u, INT_MAX};
  const auto weight = [&](int i, float z) -> unsigned long long {
    if (!kept.has(key_of<T>(z), i)) return 0;
    const float e = row_exp2(z, zmax, scale);
    return e < pmin ? 0 : weight_of(e);
  };
  const auto weight_at = [&](int i) { return weight(i, Row<T>::to_float(s.data[i - s.lo])); };
  const auto weigh = [&]() {
    unsigned long long m[1] = {0};
    for_slice(s, [&](int i, float z) { m[0] += weight(i, z); });
    parts = exchange_sums(c, m);
    whole = parts.sum(ctas, 0);
  };
  // Of the elements that `tie` names, the index of the need-th.
  const auto nth_tie = [&](uint32_t need, auto&& tie) {
    unsigned long long m[1] = {0};
    for (int i = s.lo + threadIdx.x; i < s.hi; i += blockDim.x) m[0] += tie(i);
    const Parts tied = exchange_sums(c, m);
    return tell_index(c, find_index(c, s, tied.of(0), need - 1, tie));
  };
  if (k > 0) {
    const Cut cut = find_cut<false>(c, top, k, [&](auto&& f) {
      for_slice(s, [&](int i, float z) {
        if (i >= s.lo && i < s.hi) f(key_of<T>(z), 0ull);
      });
    });
    int last = INT_MAX;
    const uint32_t need = k - cut.above.count;  // of the elements with the cut's key
    if (need < cut.at.count)
      last = nth_tie(need, [&](int i) -> unsigned long long {
        return key_of<T>(Row<T>::to_float(s.data[i - s.lo])) == cut.key;
      });
    kept = Kept{cut.key, last};
    weigh();
  }
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
    if (need < cut.at.count)
      last = nth_tie(static_cast<uint32_t>(need), [&](int i) -> unsigned long long {
        return key_of<T>(Row<T>::to_float(s.data[i - s.lo])) == cut.key && weight_at(i) != 0;
      });
    if (cut.key == kept.key) last = min(last, kept.last);
    kept = Kept{cut.key, last};
    weigh();
  }
  unsigned long long drawn =
      static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(whole));
  if (drawn > whole - 1) drawn = whole - 1;
  const int ix = find_index(c, s, parts.of(0), drawn, weight_at);
  if (ix >= 0) {
    p.token[r] = ix;
    p.prob[r] = static_cast<float>(static_cast<double>(weight_at(ix)) / static_cast<double>(whole));
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

template <typename T>
__global__ void __launch_bounds__(kRowMaxThreads)
    top_rows_kernel(const __grid_constant__ TopParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  row_begin();
  RowCta c{&sh, static_cast<int>(cluster_ctarank()), ctas, 0};
  const int r = blockIdx.x / ctas;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T> s = row_slice(row, p.V, c.rank, ctas, slice_smem);
  if (threadIdx.x == 0) sh.listed = 0;
  const float thread_max = load_row(s, row);
  row_begun();
  const Floor floor = row_floor<T>(c, thread_max, p.V <= kListMax ? 0 : p.K);
  const float zmax = floor.zmax;
  const float scale = __fdiv_rn(kRowLog2e, p.temperature);
  const float low = floor.low<T>();
  // A row of small size is listed whole; a NaN is above every floor.
  bool listing = p.V <= kListMax || floor.key > 0;
  float sum = 0.0f;
  uint32_t pushed = 0;
  for (int v = threadIdx.x; v < s.n_vec; v += blockDim.x) {
    float z[kVec];
    Row<T>::unpack(s.vec[v], z);
    bool any = false;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      sum += fast_exp2((z[e] - zmax) * scale);
      any |= !(z[e] < low);
    }
    if (listing && any) pushed += push_vector(c, s, v, z, floor.key);
  }
  sum = __uint_as_float(
      static_cast<uint32_t>(cta_reduce(c, __float_as_uint(sum), AddFloatOp(), 1)));
  const unsigned long long v[2] = {cta_reduce(c, pushed, AddOp()), __float_as_uint(sum)};
  const Parts parts = cluster_exchange(c, v);
  sum = __uint_as_float(static_cast<uint32_t>(parts.of(1)[0]));
  for (int q = 1; q < ctas; ++q) sum += __uint_as_float(static_cast<uint32_t>(parts.of(1)[q]));
  unsigned long long n = parts.sum(ctas, 0);
  listing = listing && n <= kListMax;
  if (!listing) {
    // Too many equal or too few threads: search for the K-th key, list the K.
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
      unsigned long long m[1] = {0};
      for (int i = s.lo + threadIdx.x; i < s.hi; i += blockDim.x) m[0] += tie(i);
      const Parts tied = exchange_sums(c, m);
      kept.last = tell_index(c, find_index(c, s, tied.of(0), need - 1, tie));
    }
    if (threadIdx.x == 0) sh.listed = 0;
    row_sync();  // nobody reads the bins of the search any more: the list lies over them
    for_slice(s, [&](int i, float z) {
      const uint32_t key = key_of<T>(z);
      if (i >= s.lo && i < s.hi && kept.has(key, i)) push_candidate(c, key, i);
    });
    n = p.K;
    row_sync();
  }
  if (c.rank != 0) return;  // nothing is written into the other CTAs any more
  cta_sort_any(sh.list, static_cast<int>(n));
  for (int i = threadIdx.x; i < p.K; i += blockDim.x) {
    const unsigned long long x = sh.list[i];
    p.values[static_cast<long long>(r) * p.K + i] = value_of_key<T>(candidate_key(x));
    p.index[static_cast<long long>(r) * p.K + i] = candidate_index(x);
  }
  if (threadIdx.x == 0) {
    const float inf = __uint_as_float(0x7f800000u);
    p.lse[r] = fabsf(zmax) < inf ? __fdiv_rn(zmax, p.temperature) + logf(sum) : zmax;
  }
}

}  // namespace cai
