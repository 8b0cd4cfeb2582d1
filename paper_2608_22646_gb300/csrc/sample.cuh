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
constexpr float kLn2 = 0.6931471805599453f;
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

// 2^x of a logit relative to the largest.  Subtraction and product are rounded
// one by one, as the definition says.
__device__ __forceinline__ float row_exp2(float z, float zmax, float scale) {
  return exp2f(__fmul_rn(__fsub_rn(z, zmax), scale));
}
// 2^x of a pair of logits relative to the largest, bit for bit row_exp2 where a
// weight remains.
__device__ __forceinline__ float2 row_exp2_pair(float z0, float z1, float zmax, float scale) {
  const float2 x = __fmul2_rn(__fadd2_rn(make_float2(z0, z1), make_float2(-zmax, -zmax)),
                              make_float2(scale, scale));
  return make_float2(fast_exp2(x.x), fast_exp2(x.y));
}

// Elements above a value, and of those with that value the ones up to an index.
struct Kept {
  float value;
  int last;
  __device__ __forceinline__ bool has(float z, int i) const {
    return z > value || (z == value && i <= last);
  }
};

// The row's largest logit, and a key with at least `want` elements of the row at
// or above it (0: none is known): every warp finds one for its part of them.
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
// full: the warps of a CTA whose lanes all have elements, one at least; where there
// are fewer than warps, they alone find it.
template <typename T, typename C>
__device__ __forceinline__ Floor row_floor(C& c, const Maxima<T>& m, int want, int full) {
  const int warps = c.ctas() * full;
  uint32_t floor = 0;
  if (want > 0)
    floor = static_cast<int>(threadIdx.x >> 5) < full ? warp_floor<T>(m, (want + warps - 1) / warps) : 0xffffffffu;
  // Both as one value: the largest key, and the smallest floor as its complement.
  const uint32_t top = __reduce_max_sync(0xffffffffu, key_of<float>(m.all()));
  RowShared* sh = c.sh;
  const int lane = threadIdx.x & 31, n = blockDim.x >> 5;
  if (lane == 0) sh->wred[0][threadIdx.x >> 5] = (static_cast<unsigned long long>(top) << 32) | floor;
  __syncthreads();
  const unsigned long long w = sh->wred[0][lane & (n - 1)];
  const unsigned long long v[1] = {
      (static_cast<unsigned long long>(__reduce_max_sync(0xffffffffu, static_cast<uint32_t>(w >> 32))) << 32) |
      __reduce_min_sync(0xffffffffu, static_cast<uint32_t>(w))};
  const unsigned long long* parts = cluster_exchange(c, v).of(0);
  uint32_t key = static_cast<uint32_t>(parts[0]), high = static_cast<uint32_t>(parts[0] >> 32);
#pragma unroll 1
  for (int i = 1; i < c.ctas(); ++i) {
    high = max(high, static_cast<uint32_t>(parts[i] >> 32));
    key = min(key, static_cast<uint32_t>(parts[i]));
  }
  return Floor{value_of_key<float>(high), key};
}

// How a row's weights are drawn from.
struct Setting {
  float zmax, scale, pmin, share, u;
  int k;
  __device__ __forceinline__ unsigned long long target(unsigned long long whole) const {
    const unsigned long long t = static_cast<unsigned long long>(
        ceil(static_cast<double>(share) * static_cast<double>(whole)));
    return t < 1 ? 1 : t > whole ? whole : t;
  }
  __device__ __forceinline__ float share_of(float z) const {
    const float e = row_exp2(z, zmax, scale);
    return e < pmin ? 0.0f : e;
  }
  __device__ __forceinline__ unsigned long long weight(float z) const {
    return weight_of(share_of(z));
  }
};

// The shares of two elements (find_index): of all that min-p leaves, and of those
// of them that are kept.  Handed on as values: what is handed on by reference
// lies in memory and is read again for every vector.
struct ShareAll {
  float zmax, scale, pmin;
  __device__ __forceinline__ explicit ShareAll(const Setting& s) : zmax(s.zmax), scale(s.scale), pmin(s.pmin) {}
  __device__ __forceinline__ float2 operator()(int, float z0, float z1) const {
    float2 e = row_exp2_pair(z0, z1, zmax, scale);
    e.x = e.x < pmin ? 0.0f : e.x;
    e.y = e.y < pmin ? 0.0f : e.y;
    return e;
  }
};
struct ShareKept {
  ShareAll all;
  Kept kept;
  __device__ __forceinline__ float2 operator()(int i, float z0, float z1) const {
    float2 e = all(i, z0, z1);
    e.x = kept.has(z0, i) ? e.x : 0.0f;
    e.y = kept.has(z1, i + 1) ? e.y : 0.0f;
    return e;
  }
};
// Of the elements with one key that have a share, each one unit.
template <typename T, typename Share>
struct ShareTies {
  Share share;
  uint32_t key;
  int lo, hi;
  __device__ __forceinline__ float2 operator()(int i, float z0, float z1) const {
    const float2 e = share(i, z0, z1);
    return make_float2(i >= lo && i < hi && key_of<T>(z0) == key && weight_of(e.x) ? kOneUnit : 0.0f,
                       i + 1 >= lo && i + 1 < hi && key_of<T>(z1) == key && weight_of(e.y) ? kOneUnit : 0.0f);
  }
};
struct ShareOne {
  __device__ __forceinline__ float2 operator()(int, float, float) const { return make_float2(1.0f, 1.0f); }
};
struct DrawnAt {  // a place known beforehand
  unsigned long long at;
  __device__ __forceinline__ unsigned long long operator()(unsigned long long) const { return at; }
};
struct DrawnNever {
  __device__ __forceinline__ unsigned long long operator()(unsigned long long whole) const { return whole; }
};
struct DrawnBy {
  float u;
  __device__ __forceinline__ unsigned long long operator()(unsigned long long whole) const {
    const unsigned long long d =
        static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(whole));
    return d < whole ? d : whole - 1;
  }
};

// The vectors of a thread (for_slice) with an element that is not below the floor,
// a bit for one or more of its rounds: the pass that looks for them only sets bits.
struct Noted {
  unsigned long long bits = 0;
  float low;
  int shift;  // of a vector's number to its bit
  __device__ __forceinline__ explicit Noted(int n_vec) : low(0.0f) {
    shift = __ffs(blockDim.x) - 1;
#pragma unroll 1
    while (n_vec >> shift >= 64) ++shift;
  }
  template <typename T>
  __device__ __forceinline__ void look(int v, const uint4& q) {
    if (!(vec_max(q, __uint_as_float(0xff800000u), T()) < low)) set(v);
  }
  __device__ __forceinline__ void set(int v) { bits |= 1ull << (v >> shift); }
};

// After the pass, pushes the elements that are not below the floor, each thread
// some of the noted vectors of all, and calls f(value) for each.  Returns how many
// this thread pushed; more than the list holds if there were too many vectors.
// again: they were noted above a lower floor than the final one; should they be too
// many, the row is looked through once more (500 rows of 152064 float32, K = 64: 103
// us; searching for the K-th instead 199).
template <typename T, typename C, typename S, typename F>
__device__ __forceinline__ uint32_t push_noted(const C& c, const S& s, Noted noted, bool again, F&& f) {
  RowShared* sh = c.sh;
  const int nt = blockDim.x, tid = threadIdx.x;
  const int first = S::kKept ? 0 : s.first, last = S::kKept ? s.n_vec : s.last;
  const int span = (1 << noted.shift) / nt;  // rounds of a bit
  const int end = S::kKept ? -1 : s.end_of(tid);
  uint32_t n;
#pragma unroll 1
  for (;;) {
    const uint32_t mine = __popcll(noted.bits) * span + (end >= 0);
    if (mine) {
      uint32_t at = atomicAdd(&sh->noted, mine);
      if (end >= 0 && at < kListMax) sh->note[at++] = static_cast<uint32_t>(end);
      unsigned long long bits = noted.bits;
#pragma unroll 1
      while (bits) {
        const int k = __ffsll(bits) - 1;
        bits &= bits - 1;
#pragma unroll 1
        for (int j = 0; j < span; ++j, ++at) {
          // (what an end set stands for one of the thread's other vectors)
          const int v = (k * span + j) * nt + tid;
          if (at < kListMax) sh->note[at] = v >= first && v < last ? static_cast<uint32_t>(v) : ~0u;
        }
      }
    }
    __syncthreads();
    n = sh->noted;
    if (n <= kListMax) break;
    if (!again) return kListMax + 1;
    again = false;
    __syncthreads();  // read by all
    if (tid == 0) sh->noted = 0;
    noted.bits = 0;
    for_slice<4>(s, [&](int v, const uint4& q) { noted.look<T>(v, q); });
    __syncthreads();
  }
  uint32_t pushed = 0;
#pragma unroll 1
  for (uint32_t k = tid; k < n; k += nt) {
    const uint32_t v = sh->note[k];
    if (v == ~0u) continue;
    float z[Row<T>::kVec];
    Row<T>::unpack(s.get(v), z);
#pragma unroll
    for (int e = 0; e < Row<T>::kVec; ++e) {
      const int i = s.index(v) + e;
      if (!(z[e] < noted.low) && s.holds(i)) {
        push_candidate(c, key_of<T>(z[e]), i);
        f(z[e]);
        ++pushed;
      }
    }
  }
  return pushed;
}

// The first pass of a row that is looked through for at least `want` largest
// elements (0: for the largest alone); returns the floor.  A CTA alone looks during
// the pass itself, above a floor from the part of the row that it keeps, and then
// through that part, above the final one: no second pass over the rest.  looked:
// whether `noted` is complete; f(vector, ref) was then called once for every
// vector, ref the largest element of the part kept.
template <typename T, bool kCluster, typename C, typename F>
__device__ __forceinline__ Floor load_row(C& c, const Slice<T, kCluster>& s, int want, bool look,
                                          Noted& noted, bool& looked, float& ref, F&& f) {
  const int warps = static_cast<int>(blockDim.x >> 5);
  Maxima<T> m;
  looked = false;
  if (!kCluster && look && s.keep > 0) {
    load_part<4>(s, 0, s.keep, [&](int, const uint4& v) { m.add(v); });
    const uint32_t mine = warp_floor<T>(m, (want + warps - 1) / warps);
    const uint32_t top = __reduce_max_sync(0xffffffffu, key_of<float>(m.all()));
    unsigned long long* found = c.sh->wred[1];
    if ((threadIdx.x & 31) == 0) found[threadIdx.x >> 5] = (static_cast<unsigned long long>(top) << 32) | mine;
    __syncthreads();
    const unsigned long long w = found[threadIdx.x & (warps - 1)];
    const uint32_t key = __reduce_min_sync(0xffffffffu, static_cast<uint32_t>(w));
    ref = value_of_key<float>(__reduce_max_sync(0xffffffffu, static_cast<uint32_t>(w >> 32)));
    noted.low = Floor{0.0f, key}.low<T>();
    looked = key > 0;
  }
  if (looked) {
    load_part<4>(s, s.keep, s.n_vec, [&](int v, const uint4& q) {
      if (!(m.add(q) < noted.low)) noted.set(v);
      f(q, ref);
    });
  } else {
    load_part<4>(s, !kCluster && look ? s.keep : 0, s.n_vec, [&](int, const uint4& v) { m.add(v); });
  }
  load_ends(s, [&](int, const uint4& v) {
    m.add(v);
    if (looked) f(v, ref);
  });
  c.begun();
  // (slices of several CTAs are long)
  const int full = c.ctas() > 1 ? warps : max(1, min(warps, s.last / 32));
  const Floor floor = row_floor<T>(c, m, want, full);
  noted.low = floor.low<T>();
  if (looked)
    for_body<4>(s, threadIdx.x, s.keep, blockDim.x, [&](int v, const uint4& q) {
      noted.look<T>(v, q);
      f(q, ref);
    });
  return floor;
}

// Every element of the slice, as f(index, value).
template <typename T, typename S, typename F>
__device__ __forceinline__ void for_elements(const S& s, F&& f) {
  for_slice<2>(s, [&](int v, const uint4& r) {
    float z[Row<T>::kVec];
    Row<T>::unpack(r, z);
#pragma unroll
    for (int e = 0; e < Row<T>::kVec; ++e)
      if (s.holds(s.index(v) + e)) f(s.index(v) + e, z[e]);
  });
}

// The last element kept, found by one thread of the row: for all.
template <typename T, typename C>
__device__ __forceinline__ Kept tell_kept(const C& c, bool mine, unsigned long long x) {
  const Told t = tell(c, mine, candidate_key(x), static_cast<uint32_t>(candidate_index(x)));
  return Kept{value_of_key<T>(t.a), static_cast<int>(t.b)};
}

// Of the elements with key `key` that have a share, the need-th by index is the
// last one kept.
template <typename T, typename C, typename S, typename Share>
__device__ __forceinline__ Kept keep_ties(C& c, const S& s, uint32_t key, unsigned long long need,
                                          const Share& share) {
  unsigned long long whole, found;
  const int at = find_index<T>(c, s, ShareTies<T, Share>{share, key, s.lo, s.hi}, DrawnAt{need - 1}, whole, found);
  return tell_kept<T>(c, at >= 0, candidate(key, at));
}

// The first `want` elements of the falling order.
template <typename T, typename C, typename S>
__device__ __noinline__ Kept keep_count(C& c, const S s, uint32_t want) {
  const Cut cut = find_cut<T>(c, 0xffffffffu >> (32 - Row<T>::kKeyBits), want, kListMax, [&](auto&& f) {
    for_elements<T>(s, [&](int, float z) { f(key_of<T>(z)); });
  });
  if (cut.at > kListMax)  // one key, more often than a list holds
    return keep_ties<T>(c, s, cut.lo, want - cut.above, ShareOne{});
  // List what lies there, and look.
  if (threadIdx.x == 0) c.sh->listed = 0;
  c.sync();
  for_elements<T>(s, [&](int i, float z) {
    const uint32_t key = key_of<T>(z);
    if (key - cut.lo <= cut.hi - cut.lo) push_candidate(c, key, i);
  });
  c.sync();
  const bool mine = c.rank() == 0 && threadIdx.x == 0;
  unsigned long long x = 0;
  if (c.rank() == 0) x = cta_sort(c.sh->list, static_cast<int>(cut.at))[want - cut.above - 1];
  return tell_kept<T>(c, mine, x);
}

// What a search by weight starts from: values in [low, high] (open: below high),
// `above` the weight of what lies higher.
struct Bracket {
  float low, high;
  bool open;
  unsigned long long above;
  __device__ __forceinline__ bool holds(float z) const {
    return z >= low && (open ? z < high : z <= high);
  }
  __device__ __forceinline__ bool higher(float z) const { return open ? z >= high : z > high; }
  // kBins equal parts; rising with z.
  __device__ __forceinline__ int bin(float z) const {
    const float b = (z - low) * (static_cast<float>(kBins) / (high - low));
    return b >= static_cast<float>(kBins - 1) ? kBins - 1 : b > 0.0f ? static_cast<int>(b) : 0;
  }
};

// The first elements of the falling order whose weight reaches `want`; share(i,
// z0, z1) as in find_index, falling with the value.  First a guess: the numbers
// of elements in equal parts of the bracket, each taken with the weight at its
// middle, say in which part the cut lies; then one exact pass adds up what lies
// above it and lists its elements (and those of its neighbours, if there is room),
// and moves on where the guess was wrong.  Where they are too many for a list, the
// key is found by halving the range of keys with an exact sum each time.
template <typename T, typename C, typename S, typename Share>
__device__ __noinline__ Kept keep_weight(C& c, const S s, const Bracket br, unsigned long long want,
                                         const Share share) {
  constexpr int kVec = Row<T>::kVec;
  const auto weight_at = [&](int i, float z) { return weight_of(share(i, z, z).x); };
  // The weight of the elements that pick(i, z) names.
  const auto sum_of = [&](auto&& pick, unsigned long long also, unsigned long long& other) {
    WeightSum sum;
    uint32_t n = 0;
    for_slice<2>(s, [&](int v, const uint4& r) {
      float z[kVec];
      Row<T>::unpack(r, z);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const int i = s.index(v) + e;
        const float2 w = share(i, z[e], z[e + 1]);
        sum.add(pick(i, z[e]) ? w.x : 0.0f, pick(i + 1, z[e + 1]) ? w.y : 0.0f);
      }
      n += kVec;
    });
    const unsigned long long m[2] = {sum.sum(n), other};
    const Parts parts = exchange_sums(c, m);
    other = parts.sum(c.ctas(), 1);
    return parts.sum(c.ctas(), 0) + also;
  };
  if (br.high > br.low && br.high - br.low < 1e30f) {
    const float width = (br.high - br.low) / kBins;
    const Level l = search_level(
        c, br.above, want,
        [&](auto&& f) {
          for_elements<T>(s, [&](int, float z) {
            if (br.holds(z)) f(br.bin(z));
          });
        },
        [&](int b, uint32_t n) -> unsigned long long {
          // (of index -1: before every element, so that ties are not cut)
          const float z = br.low + (static_cast<float>(b) + 0.5f) * width;
          return static_cast<unsigned long long>(static_cast<float>(n) * kWeightUnit * share(-1, z, z).x);
        });
    // (-1: the guesses add up to less than is wanted; then it is the lowest part)
    int bin = max(l.bin, 0);
    const int around = l.bin >= 0 && 4 * l.count < kListMax ? 1 : 0;  // parts to either side
#pragma unroll 1
    for (int turn = 0; turn < 4 && bin >= 0 && bin < kBins; ++turn) {
      if (threadIdx.x == 0) c.sh->listed = 0;
      c.sync();
      unsigned long long pushed = 0;
      const unsigned long long above = sum_of(
          [&](int i, float z) {
            if (!br.holds(z)) return false;
            const int d = br.bin(z) - bin;
            if (d <= around && d >= -around && s.holds(i) && weight_at(i, z) != 0) {
              push_candidate(c, key_of<T>(z), i);
              ++pushed;
            }
            return d > around;
          },
          br.above, pushed);
      const uint32_t n = static_cast<uint32_t>(pushed);  // of all CTAs now
      if (n > kListMax) break;
      int step = 0;  // where to look next
      bool mine = false;
      unsigned long long x = 0;
      if (above >= want) {
        step = 1;
      } else if (c.rank() == 0) {
        const unsigned long long* list = cta_sort(c.sh->list, static_cast<int>(n));
        const int nt = blockDim.x, per = (static_cast<int>(n) + nt - 1) / nt;
        const int a = min(static_cast<int>(n), static_cast<int>(threadIdx.x) * per);
        const int b = min(static_cast<int>(n), a + per);
        const auto weight_in = [&](int i) {
          return weight_at(candidate_index(list[i]), value_of_key<T>(candidate_key(list[i])));
        };
        unsigned long long own = 0, all;
#pragma unroll 1
        for (int i = a; i < b; ++i) own += weight_in(i);
        unsigned long long run = above + cta_scan(c.sh, own, all);
#pragma unroll 1
        for (int i = a; i < b && !mine && run < want; ++i) {
          run += weight_in(i);
          if (run >= want) {
            mine = true;
            x = list[i];
          }
        }
        if (above + all < want) {  // further down
          mine = threadIdx.x == 0;
          x = ~0ull;
        }
      }
      if (step == 0) {
        const Told t = tell(c, mine, candidate_key(x), static_cast<uint32_t>(candidate_index(x)));
        if (static_cast<int>(t.b) >= 0) return Kept{value_of_key<T>(t.a), static_cast<int>(t.b)};
        step = -1;
      }
      bin += step * (2 * around + 1);
      c.sync();  // the list and what was told have been read
    }
  }
  // The largest key with enough weight at or above it.
  uint32_t key = 0;
  unsigned long long none = 0;
#pragma unroll 1
  for (int bit = Row<T>::kKeyBits - 1; bit >= 0; --bit) {
    const uint32_t t = key | (1u << bit);
    if (sum_of([&](int, float z) { return key_of<T>(z) >= t; }, 0, none) >= want) key = t;
  }
  const unsigned long long above = sum_of([&](int, float z) { return key_of<T>(z) > key; }, 0, none);
  // The same weight for every element with that key.
  const unsigned long long each = weight_at(-1, value_of_key<T>(key));
  return keep_ties<T>(c, s, key, (want - above + each - 1) / each, share);
}

// In CTA 0, with n tokens listed as (index, key): draws one of them.
template <typename T>
__device__ __forceinline__ void draw_listed(RowShared* sh, const SampleParams& p, int r, int n,
                                            const Setting& set) {
  const int tid = threadIdx.x, nt = blockDim.x;
  const auto weight = [&](unsigned long long x) {
    return set.weight(value_of_key<T>(static_cast<uint32_t>(x)));
  };
  const unsigned long long* list = cta_sort(sh->list, n);
  const int per = (n + nt - 1) / nt;
  const int a = min(n, tid * per), b = min(n, a + per);
  unsigned long long own = 0, all;
#pragma unroll 1
  for (int i = a; i < b; ++i) own += weight(list[i]);
  unsigned long long run = cta_scan(sh, own, all);
  const unsigned long long drawn = cta_once(sh, [&]() { return DrawnBy{set.u}(all); });
  if (drawn < run || drawn >= run + own) return;
#pragma unroll 1
  for (int i = a; i < b; ++i) {
    const unsigned long long w = weight(list[i]);
    run += w;
    if (drawn < run) {
      p.token[r] = static_cast<int32_t>(list[i] >> 32);
      p.prob[r] = __fdiv_rn(static_cast<float>(w), static_cast<float>(all));
      return;
    }
  }
}

// In CTA 0, with at most kListMax / 2 candidates listed (a sorted list then leaves
// that half of the room free): sorts them, keeps, draws.  `whole`: the
// weight of all tokens that min-p leaves, where top-k is off.
template <typename T>
__device__ __noinline__ void sample_candidates(RowShared* sh, const SampleParams& p, int r, int n,
                                               const Setting set, unsigned long long whole) {
  const int tid = threadIdx.x, nt = blockDim.x;
  const auto weight = [&](uint32_t key) { return set.weight(value_of_key<T>(key)); };
  unsigned long long* list = cta_sort(sh->list, n);
  if (set.k > 0) n = min(n, set.k);
  if (!(set.share < 1.0f)) {
    // All of them; those without a weight are never drawn.
#pragma unroll 1
    for (int i = tid; i < n; i += nt)
      sh->list[i] = (static_cast<unsigned long long>(candidate_index(list[i])) << 32) | candidate_key(list[i]);
    draw_listed<T>(sh, p, r, n, set);
    return;
  }
  const int per = (n + nt - 1) / nt;
  const int a = min(n, tid * per), b = min(n, a + per);
  unsigned long long own = 0, all;
#pragma unroll 1
  for (int i = a; i < b; ++i) own += weight(candidate_key(list[i]));
  const unsigned long long before = cta_scan(sh, own, all);
  unsigned long long run = before;
  if (set.k > 0) whole = all;
  // Kept are those before which the running weight is below the target.
  const unsigned long long target = cta_once(sh, [&]() { return set.target(whole); });
  int kept = 0;
#pragma unroll 1
  for (int i = a; i < b; ++i) {
    const unsigned long long w = weight(candidate_key(list[i]));
    kept += w != 0 && run < target;
    run += w;
  }
  // (weights fall along the list; should two of them not, by a rounding of 2^x at
  // min-p, what is kept is still the number of those that pass)
  unsigned long long n_kept;
  int at = static_cast<int>(cta_scan(sh, kept, n_kept));
  run = before;
#pragma unroll 1
  for (int i = a; i < b; ++i) {
    const unsigned long long x = list[i], w = weight(candidate_key(x));
    // In index order from here on, the key behind it.
    if (w != 0 && run < target)
      sh->list[at++] = (static_cast<unsigned long long>(candidate_index(x)) << 32) | candidate_key(x);
    run += w;
  }
  draw_listed<T>(sh, p, r, static_cast<int>(n_kept), set);
}

// Candidates asked for where only the weight limits what is kept (64 rows of 50003
// float32, top-p, where a nucleus has some dozens of tokens: 64 18.5 us, 128 20.5,
// 256 25; one that reaches past the listed ones takes 40 to 75 in keep_weight).
constexpr int kNucleusWant = 128;

// One pass over a row for its maximum and a floor, one for the weights (top-k needs
// none) and the candidates; few rows keep the row in shared memory, so HBM is read
// once.  Few rows are bound by the chain of reductions between the CTAs (one row of
// 126464 bf16 15 us, of which the host's call 8; 64 of 50003 float32 20 to 41), many
// by the instructions of the weights, 75 to 130 for 16 bytes, and by loads that two
// CTAs on an SM do not wholly hide: 2048 rows of 126464 bf16, settings of all kinds,
// 314 us, 1.65 TB/s.
template <typename T, bool kCluster>
__global__ void __launch_bounds__(512, kCluster ? 1 : 2)
    sample_rows_kernel(const __grid_constant__ SampleParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  using Cta = RowCta<kCluster>;
  Cta::begin();
  Cta c(&sh, ctas);
  const int r = kCluster ? blockIdx.x / ctas : blockIdx.x;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T, kCluster> s =
      row_slice<T, kCluster>(row, p.V, c.rank(), c.ctas(), slice_smem, kCluster ? 0 : ctas, sh.edge);
  if (threadIdx.x == 0) sh.listed = sh.noted = 0;
  const float inf = __uint_as_float(0x7f800000u);
  const float t = p.temperature ? p.temperature[r] : 1.0f;
  const bool greedy = !(t > 0.0f);
  Setting set;
  set.scale = greedy ? kRowLog2e : fminf(fmaxf(__fdiv_rn(kRowLog2e, t), 1e-38f), 3e38f);
  set.pmin = p.min_p ? fminf(p.min_p[r], 1.0f) : 0.0f;
  set.k = p.top_k ? p.top_k[r] : 0;
  if (set.k >= p.V || set.k < 0) set.k = 0;
  set.share = p.top_p ? p.top_p[r] : 1.0f;
  set.u = p.u[r] > 0.0f ? fminf(p.u[r], 1.0f) : 0.0f;  // NaN: 0
  // Tokens that decide the row, if a list can hold them.
  const int want = greedy ? 0
                   : set.k > 0 ? (set.k <= kListMax / 4 ? set.k : 0)
                   : set.share < 1.0f || set.pmin > 0.0f ? kNucleusWant : 0;

  Noted noted(s.n_vec);
  bool looked;
  float ref;
  const Floor floor = load_row<T, kCluster>(c, s, want, want > 0 && set.k > 0, noted, looked, ref,
                                            [](const uint4&, float) {});
  const float zmax = set.zmax = floor.zmax;

  if (!(fabsf(zmax) < inf) || greedy) {
    // The first of the largest logits; a row without a softmax has no probability.
    const bool valid = fabsf(zmax) < inf;
    int first = INT_MAX;
    WeightSum sum;
    uint32_t n = 0;
    for_slice<4>(s, [&](int v, const uint4& q) {
      float z[kVec];
      Row<T>::unpack(q, z);
      if (!(vec_max(q, -inf, T()) < zmax)) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (z[e] == zmax && s.holds(s.index(v) + e)) first = min(first, s.index(v) + e);
      }
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const float2 w = row_exp2_pair(z[e], z[e + 1], zmax, set.scale);
        sum.add(w.x, w.y);
      }
      n += kVec;
    });
    first = __reduce_min_sync(0xffffffffu, first);
    const unsigned long long ix =
        cta_reduce(&sh, first, [](unsigned long long a, unsigned long long b) { return a < b ? a : b; }, 1);
    const unsigned long long v[2] = {cta_reduce(&sh, sum.sum(n), AddOp()), ix};
    const Parts parts = cluster_exchange(c, v);
    if (c.rank() == 0 && threadIdx.x == 0) {
      unsigned long long best = parts.of(1)[0];
#pragma unroll 1
      for (int q = 1; q < c.ctas(); ++q) best = min(best, parts.of(1)[q]);
      p.token[r] = best < static_cast<unsigned long long>(p.V) ? static_cast<int>(best) : 0;
      p.prob[r] = valid ? __fdiv_rn(kWeightUnit, static_cast<float>(parts.sum(c.ctas(), 0)))
                        : __uint_as_float(0x7fc00000u);
    }
    return;  // no CTA writes into another from here on
  }

  Kept kept{-inf, INT_MAX};
  const ShareAll share_all(set);
  unsigned long long mass;
  int ix;
  Bracket br{-3e38f, zmax, false, 0};
  unsigned long long whole = 0;
  if (want > 0) {
    // One pass: the weight of every token that min-p leaves (not needed under
    // top-k), and the candidates.
    const bool listing = p.V <= kListMax || floor.key > 0;
    const float low = noted.low;
    WeightSum sum;
    uint32_t n = 0, pushed = 0;
    unsigned long long listed_mass = 0;
    if (set.k > 0) {
      if (listing && !looked)
        for_slice<4>(s, [&](int v, const uint4& q) { noted.look<T>(v, q); });
    } else {
      for_slice<4>(s, [&](int v, const uint4& q) {
        float z[kVec];
        Row<T>::unpack(q, z);
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
          float2 w = row_exp2_pair(z[e], z[e + 1], zmax, set.scale);
          w.x = w.x < set.pmin ? 0.0f : w.x;
          w.y = w.y < set.pmin ? 0.0f : w.y;
          sum.add(w.x, w.y);
        }
        n += kVec;
        if (listing) noted.look<T>(v, q);
      });
    }
    if (listing)
      pushed = push_noted<T>(c, s, noted, looked, [&](float z) {
        if (set.k == 0) listed_mass += set.weight(z);
      });
    const unsigned long long sums[3] = {sum.sum(n), listed_mass, pushed};
    const Parts parts = exchange_sums(c, sums);
    whole = parts.sum(c.ctas(), 0);
    const unsigned long long target =
        set.k == 0 && set.share < 1.0f ? cta_once(&sh, [&]() { return set.target(whole); }) : whole;
    const unsigned long long n_listed = parts.sum(c.ctas(), 2);
    if (listing && n_listed <= kListMax / 2) {
      // All that is kept is listed: the first k; or enough weight for the target;
      // or everything that has a weight.
      const unsigned long long mass = parts.sum(c.ctas(), 1);
      if (set.k > 0 || mass >= target) {
        if (c.rank() == 0) sample_candidates<T>(&sh, p, r, static_cast<int>(n_listed), set, whole);
        return;
      }
    }
    if (set.k == 0 && set.share < 1.0f) {
      // The cut lies below the listed ones or, where they are too many for a list
      // but heavy enough, among them; and above what could hold no more than the
      // rest of the weight were every token that light.
      const unsigned long long light = (whole - target) / p.V;
      const float e = fmaxf(static_cast<float>(light) - 0.5f, 0.5f) * kOneUnit * 0.99f;
      br.low = fmaxf(zmax + log2f(fmaxf(e, 0.99f * set.pmin)) / set.scale - 1e-3f * fabsf(zmax), -3e38f);
      if (listing && low > -inf && n_listed <= kListMax) {  // their weight is known
        const unsigned long long above = parts.sum(c.ctas(), 1);
        if (above < target) {
          br.high = low;
          br.open = true;
          br.above = above;
        } else {
          br.low = fmaxf(br.low, low);
        }
      }
    }
  }
  if (set.k > 0) {
    kept = keep_count<T>(c, s, set.k);
    if (set.share < 1.0f) {
      find_index<T>(c, s, ShareKept{share_all, kept}, DrawnNever{}, whole, mass);  // the sum alone
      br.low = kept.value;
    }
  }
  if (set.share < 1.0f)
    kept = keep_weight<T>(c, s, br, cta_once(&sh, [&]() { return set.target(whole); }),
                          ShareKept{share_all, kept});
  if (set.k > 0 || set.share < 1.0f)
    ix = find_index<T>(c, s, ShareKept{share_all, kept}, DrawnBy{set.u}, whole, mass);
  else
    ix = find_index<T>(c, s, share_all, DrawnBy{set.u}, whole, mass);
  if (ix >= 0) {
    p.token[r] = ix;
    p.prob[r] = __fdiv_rn(static_cast<float>(mass), static_cast<float>(whole));
  }
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

// The maximum and a floor, the sum of exponentials, the candidates sorted.  32 rows
// of 152064 bf16, K = 64: 15 us, bound by latency and the host's call; 2000 of
// 126464, K = 128: 177 us, 2.9 TB/s of 506 MB read once.  The SMs issue on 55 % of
// the cycles: 60 instructions for 16 bytes and some 20000 a row for floors, pushes
// and the sort, whose barriers and loads two CTAs on an SM hide in part only.
template <typename T, bool kCluster>
__global__ void __launch_bounds__(512, kCluster ? 1 : 2)
    top_rows_kernel(const __grid_constant__ TopParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  using Cta = RowCta<kCluster>;
  Cta::begin();
  Cta c(&sh, ctas);
  const int r = kCluster ? blockIdx.x / ctas : blockIdx.x;
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  const Slice<T, kCluster> s =
      row_slice<T, kCluster>(row, p.V, c.rank(), c.ctas(), slice_smem, kCluster ? 0 : ctas, sh.edge);
  if (threadIdx.x == 0) sh.listed = sh.noted = 0;
  const float inf = __uint_as_float(0x7f800000u);
  const float scale = __fdiv_rn(kRowLog2e, p.temperature);
  // The sum of 2^((z - base) scale).  A CTA alone takes it along in the first pass,
  // with base the largest element of the part that it keeps: one fused step, without
  // a running maximum (2000 rows of 126464 bf16, K = 128: with one in each thread,
  // which nearly every vector raises somewhere in a warp, 185 us; so 176).  x =
  // z scale - fl(base scale) is off by that product's rounding, which comes off the
  // sum's logarithm.
  float2 sum2 = make_float2(0.0f, 0.0f);
  float base;
  Noted noted(s.n_vec);
  bool looked;
  const Floor floor = load_row<T, kCluster>(
      c, s, p.K, true, noted, looked, base, [&](const uint4& q, float ref) {
        const float from = -__fmul_rn(ref, scale);
        float z[kVec];
        Row<T>::unpack(q, z);
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
          const float2 x = __ffma2_rn(make_float2(z[e], z[e + 1]), make_float2(scale, scale), make_float2(from, from));
          sum2 = __fadd2_rn(sum2, make_float2(fast_exp2(x.x), fast_exp2(x.y)));
        }
      });
  const float zmax = floor.zmax;
  // (a NaN is above every floor)
  const bool listing = p.V <= kListMax || floor.key > 0;
  uint32_t pushed = 0;
  // Where base is far below the row's largest, or no number, or so large that the
  // product's rounding moves the sum by more than a few binary places (a row at its
  // type's lowest value: by 10^30 of them), the sum is taken again.
  float off = looked ? -__fmaf_rn(base, scale, -__fmul_rn(base, scale)) : 0.0f;
  const bool summed = looked && !__syncthreads_or(!(sum2.x + sum2.y < 1.15e18f && fabsf(off) < 8.0f));
  if (!summed) {
    off = 0.0f;
    base = zmax;
    sum2 = make_float2(0.0f, 0.0f);
    for_slice<4>(s, [&](int v, const uint4& q) {
      float z[kVec];
      Row<T>::unpack(q, z);
#pragma unroll
      for (int e = 0; e < kVec; e += 2)
        sum2 = __fadd2_rn(sum2, row_exp2_pair(z[e], z[e + 1], base, scale));
      if (listing && !looked) noted.look<T>(v, q);
    });
  }
  if (listing) pushed = push_noted<T>(c, s, noted, looked, [](float) {});
  float sum = __uint_as_float(static_cast<uint32_t>(
      cta_reduce(&sh, __float_as_uint(sum2.x + sum2.y), AddFloatOp(), 1)));
  const unsigned long long v[2] = {
      cta_reduce(&sh, pushed, AddOp()), __float_as_uint(sum)};
  const Parts parts = cluster_exchange(c, v);
  sum = __uint_as_float(static_cast<uint32_t>(parts.of(1)[0]));
#pragma unroll 1
  for (int q = 1; q < c.ctas(); ++q) sum += __uint_as_float(static_cast<uint32_t>(parts.of(1)[q]));
  uint32_t n = static_cast<uint32_t>(parts.sum(c.ctas(), 0));
  if (!listing || n > kListMax) {
    // Too many equal or too few threads: search for the K-th, list the K.
    const Kept kept = keep_count<T>(c, s, p.K);
    if (threadIdx.x == 0) sh.listed = 0;
    c.sync();
    const uint32_t cut = key_of<T>(kept.value);
    for_elements<T>(s, [&](int i, float z) {
      const uint32_t key = key_of<T>(z);
      if (key > cut || (key == cut && i <= kept.last)) push_candidate(c, key, i);
    });
    n = p.K;
    c.sync();
  }
  if (c.rank() != 0) return;  // nothing is written into the other CTAs any more
  const unsigned long long* sorted = cta_sort(sh.list, static_cast<int>(n));
#pragma unroll 1
  for (int i = threadIdx.x; i < p.K; i += blockDim.x) {
    const unsigned long long x = sorted[i];
    p.values[static_cast<long long>(r) * p.K + i] = value_of_key<T>(candidate_key(x));
    p.index[static_cast<long long>(r) * p.K + i] = candidate_index(x);
  }
  if (threadIdx.x == 0)
    p.lse[r] = fabsf(zmax) < inf ? __fdiv_rn(base, p.temperature) + (logf(sum) + off * kLn2) : zmax;
}

}  // namespace cai
