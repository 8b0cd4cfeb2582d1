// What the operators on rows of vocabulary logits share: a row is cut over the
// CTAs of one thread-block cluster, each keeps its slice in shared memory for
// every pass it makes, and the cluster reduces and searches through distributed
// shared memory.  HBM is read once, and no call needs a workspace.
#pragma once

#include <climits>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"

namespace cai {

constexpr int kRowMaxCluster = 8;    // portable cluster size
constexpr int kRowMaxThreads = 512;
constexpr int kRowMaxWarps = kRowMaxThreads / 32;
constexpr int kRowSliceMax = 192 * 1024;  // bytes of a row that one CTA keeps

// A vector of 16 bytes of logits as floats.
template <typename T>
struct Row;
template <>
struct Row<float> {
  static constexpr int kVec = 4;
  static constexpr int kKeyBits = 32;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float to_float(float x) { return x; }
  static __device__ __forceinline__ float from_float(float x) { return x; }
  static __device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }
};
template <>
struct Row<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static constexpr int kKeyBits = 16;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 from_float(float x) {
    return __float2bfloat16_rn(x);
  }
  static __device__ __forceinline__ __nv_bfloat16 neg_inf() {
    return __ushort_as_bfloat16(static_cast<unsigned short>(0xff80u));
  }
};

// max that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The largest of a vector and of `m`, NaN kept.
__device__ __forceinline__ float vec_max(const uint4& v, float m, float) {
  m = max_nan(m, max_nan(__uint_as_float(v.x), __uint_as_float(v.y)));
  return max_nan(m, max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float vec_max(const uint4& v, float m, __nv_bfloat16) {
  const uint32_t r = max2_nan(max2_nan(v.x, v.y), max2_nan(v.z, v.w));
  return max_nan(m, max_nan(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)));
}

// Order of the logits as whole numbers: rises with the value, -0 and +0 are the
// same, NaN is above +inf.  bf16 values differ in the upper 16 bits alone.
template <typename T>
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);
  uint32_t k = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
  if (z != z) k = 0xffffffffu;
  return Row<T>::kKeyBits == 16 ? k >> 16 : k;
}
template <typename T>
__device__ __forceinline__ float value_of_key(uint32_t k) {
  if (Row<T>::kKeyBits == 16) k = (k << 16) | (k & 0x8000u ? 0u : 0xffffu);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// The slice of a row that this CTA keeps: elements [lo, hi) of the row, element
// lo + i at data[i].  The bytes lie in shared memory as they do in global memory
// modulo 16, so whole 16-byte vectors are copied as such; what a first or last
// vector holds besides the slice is -inf.  A vector v covers the elements
// lo - skip + v kVec ...
template <typename T>
struct Slice {
  uint4* vec;   // vectors of the slice
  int n_vec;
  T* data;
  int lo, hi;   // elements of the row
  int skip;     // elements of the first vector before the slice

  __device__ __forceinline__ int index(int v, int e) const {
    return lo - skip + v * Row<T>::kVec + e;
  }
  __device__ __forceinline__ int pads() const { return n_vec * Row<T>::kVec - (hi - lo); }
};

// Elements per CTA of a row of V over `ctas`: a multiple of 64.
__host__ __device__ __forceinline__ int row_chunk(int V, int ctas) {
  return ((V + ctas - 1) / ctas + 63) / 64 * 64;
}
// Shared memory of a slice, with room for the shifted start.
__host__ __device__ __forceinline__ size_t row_slice_bytes(int V, int ctas, int elem) {
  return static_cast<size_t>(row_chunk(V, ctas)) * elem + 32;
}

template <typename T>
__device__ __forceinline__ Slice<T> row_slice(const T* row, int V, int rank, int ctas, void* smem) {
  Slice<T> s;
  const int chunk = row_chunk(V, ctas);
  s.lo = min(V, rank * chunk);
  s.hi = min(V, s.lo + chunk);
  const uint32_t a = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + s.lo)) & 15u;
  s.skip = static_cast<int>(a / sizeof(T));
  s.vec = static_cast<uint4*>(smem);
  s.data = reinterpret_cast<T*>(static_cast<char*>(smem) + a);
  s.n_vec = s.hi > s.lo ? (s.skip + s.hi - s.lo + Row<T>::kVec - 1) / Row<T>::kVec : 0;
  return s;
}

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

// Copies the slice from global memory, vector by vector (the first and last,
// where they are not whole, element by element), and hands every vector to
// `see` on the way.  Each thread has kFlight loads in flight.
template <typename T, int kFlight, typename F>
__device__ __forceinline__ void load_slice(const Slice<T>& s, const T* row, F&& see) {
  constexpr int kVec = Row<T>::kVec;
  // Global address of vector 0, which may begin before the slice: only whole
  // vectors are read through it.
  const uint4* src = reinterpret_cast<const uint4*>(
      reinterpret_cast<uintptr_t>(row + s.lo) & ~static_cast<uintptr_t>(15));
  const int first = s.skip ? 1 : 0;
  const int last = (s.skip + s.hi - s.lo) / kVec;  // whole vectors end here
  const int step = static_cast<int>(blockDim.x);
  for (int v0 = first + static_cast<int>(threadIdx.x); v0 < last; v0 += kFlight * step) {
    uint4 r[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (v0 + j * step < last) r[j] = ld_stream(src + v0 + j * step);
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (v0 + j * step < last) {
        s.vec[v0 + j * step] = r[j];
        see(r[j]);
      }
  }
  // The vectors at the two ends that are not whole (they may be one).
  if (threadIdx.x < 2 && s.n_vec > 0) {
    const int v = threadIdx.x == 0 ? 0 : s.n_vec - 1;
    const bool part = threadIdx.x == 0 ? first != 0 : last < s.n_vec && s.n_vec - 1 >= first;
    if (part) {
      T* d = reinterpret_cast<T*>(s.vec + v);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const int i = s.index(v, e);
        d[e] = i >= s.lo && i < s.hi ? row[i] : Row<T>::neg_inf();
      }
      see(s.vec[v]);
    }
  }
}

// ------------------------------------------------------ reductions, search --

struct Tally {  // tokens and their weight
  unsigned long long mass;
  uint32_t count;
  uint32_t pad;
};

constexpr int kBins = 1024;
constexpr int kListMax = 2048;  // candidates that one CTA finishes alone
constexpr int kSums = 3;        // values of an exchange

// Shared memory of a CTA beside its slice.
struct RowShared {
  unsigned long long wred[kSums][kRowMaxWarps];          // values per warp
  unsigned long long slots[4][kSums][kRowMaxCluster];    // values per CTA, written by the peers
  Tally parts[kRowMaxCluster];
  Tally found, found_at;  // what lies above the bin that was found, and in it
  uint32_t found_bin;
  int32_t told;           // an index one thread found, for all (tell_index)
  unsigned long long part_scan[kRowMaxWarps];
  uint32_t part_scan_n[kRowMaxWarps];
  uint32_t listed;        // candidates pushed so far (in CTA 0)
  union {
    struct {              // find_cut
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    };
    unsigned long long list[kListMax];  // candidates (in CTA 0)
  };
};

struct RowCta {
  RowShared* sh;
  int rank, ctas;
  int turn;  // which slots the next reduction uses
};

// All threads of the cluster.  Warps may arrive from loops that their lanes
// left at different times.
__device__ __forceinline__ void row_sync() {
  __syncwarp();
  cluster_sync();
}

// Peers' shared memory may be written once every CTA of the cluster has begun:
// row_begin at the top of a kernel, row_begun before the first such write (and
// before any early return).
__device__ __forceinline__ void row_begin() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void row_begun() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Writes a 64-bit value into `p`'s place in the shared memory of CTA `rank`.
__device__ __forceinline__ void st_peer(const unsigned long long* p, int rank,
                                        unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_shared(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void st_peer(const uint32_t* p, int rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_shared(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ unsigned long long ld_peer(const unsigned long long* p, int rank) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(mapa_shared(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_peer(const uint32_t* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(p, rank)) : "memory");
  return v;
}

template <typename Op>
__device__ __forceinline__ unsigned long long warp_reduce(unsigned long long v, Op op) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Reduces one value per thread over the CTA, the result in every thread.  All
// threads call it; wred is free again after the next barrier.
template <typename Op>
__device__ __forceinline__ unsigned long long cta_reduce(const RowCta& c, unsigned long long v,
                                                         Op op, int which = 0) {
  v = warp_reduce(v, op);
  const int warp = threadIdx.x >> 5, n = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) c.sh->wred[which][warp] = v;
  __syncthreads();
  unsigned long long r = c.sh->wred[which][0];
  for (int i = 1; i < n; ++i) r = op(r, c.sh->wred[which][i]);
  return r;
}

// Values per CTA to every CTA of the cluster: the slots of value `which`, in rank
// order, are valid for the next three exchanges.
struct Parts {
  const unsigned long long* slot;
  __device__ __forceinline__ const unsigned long long* of(int which) const {
    return slot + which * kRowMaxCluster;
  }
  __device__ __forceinline__ unsigned long long sum(int ctas, int which) const {
    unsigned long long r = 0;
    for (int i = 0; i < ctas; ++i) r += of(which)[i];
    return r;
  }
};
template <int kN>
__device__ __forceinline__ Parts cluster_exchange(RowCta& c, const unsigned long long (&v)[kN]) {
  unsigned long long* s = &c.sh->slots[c.turn & 3][0][0];
  c.turn++;
  if (static_cast<int>(threadIdx.x) < c.ctas) {
#pragma unroll
    for (int i = 0; i < kN; ++i) st_peer(s + i * kRowMaxCluster + c.rank, threadIdx.x, v[i]);
  }
  row_sync();
  return Parts{s};
}

template <typename Op>
__device__ __forceinline__ unsigned long long cluster_reduce(RowCta& c, unsigned long long v,
                                                             Op op) {
  const unsigned long long mine[1] = {cta_reduce(c, v, op)};
  const unsigned long long* s = cluster_exchange(c, mine).of(0);
  unsigned long long r = s[0];
  for (int i = 1; i < c.ctas; ++i) r = op(r, s[i]);
  return r;
}

struct AddOp {
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return a + b;
  }
};
// The sums of up to three values per thread, CTA by CTA, to all.
template <int kN>
__device__ __forceinline__ Parts exchange_sums(RowCta& c, const unsigned long long (&v)[kN]) {
  const int warp = threadIdx.x >> 5, n = blockDim.x >> 5;
  unsigned long long r[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    r[i] = warp_reduce(v[i], AddOp());
    if ((threadIdx.x & 31) == 0) c.sh->wred[i][warp] = r[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    r[i] = 0;
    for (int w = 0; w < n; ++w) r[i] += c.sh->wred[i][w];
  }
  return cluster_exchange(c, r);
}
struct MaxOp {
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return a > b ? a : b;
  }
};
struct MaxNanOp {  // on the bits of a float
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return __float_as_uint(max_nan(__uint_as_float(static_cast<uint32_t>(a)),
                                   __uint_as_float(static_cast<uint32_t>(b))));
  }
};

// Where a falling run over the kept elements of the row first reaches `want`
// (by count or by weight): the key there, and what lies above that key.
struct Cut {
  uint32_t key;
  Tally above;  // strictly larger keys
  Tally at;     // this key
};

// Radix search from the largest key down, kBins parts of the remaining key
// range at a time.  visit(f) calls f(key, weight) for every element that takes
// part; `top` is the largest key among them.  All threads of all CTAs call it
// with the same arguments; the whole has to reach `want`.
template <bool kByMass, typename Visit>
__device__ __forceinline__ Cut find_cut(RowCta& c, uint32_t top, unsigned long long want,
                                        Visit&& visit) {
  RowShared* sh = c.sh;
  const int tid = threadIdx.x, nt = blockDim.x;
  uint32_t lo = 0, hi = top;  // the key is in [lo, hi]
  Tally above{0, 0, 0};
  for (;;) {
    const uint32_t range = hi - lo;
    const int bits = 32 - __clz(range);  // 0 for one key
    const int shift = bits > 10 ? bits - 10 : 0;
    for (int i = tid; i < kBins; i += nt) {
      sh->mass[i] = 0;
      sh->count[i] = 0;
    }
    __syncthreads();
    visit([&](uint32_t key, unsigned long long w) {
      if (key - lo <= range) {
        const uint32_t b = (key - lo) >> shift;
        atomicAdd(&sh->count[b], 1u);
        if (kByMass) atomicAdd(&sh->mass[b], w);
      }
    });
    row_sync();
    // Every CTA sums its share of the bins over the cluster; bins fall with
    // the thread index so that a rising scan runs from the largest key down.
    const int share = kBins / c.ctas;
    const int per = (share + nt - 1) / nt;  // bins of a thread
    Tally mine{0, 0, 0};
    for (int j = 0; j < per; ++j) {
      const int k = tid * per + j;
      if (k < share) {
        const int b = kBins - 1 - (c.rank * share + k);
        for (int r = 0; r < c.ctas; ++r) {
          mine.count += ld_peer(&sh->count[b], r);
          if (kByMass) mine.mass += ld_peer(&sh->mass[b], r);
        }
      }
    }
    Tally incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long m = __shfl_up_sync(0xffffffffu, incl.mass, o);
      const uint32_t n = __shfl_up_sync(0xffffffffu, incl.count, o);
      if ((tid & 31) >= o) {
        incl.mass += m;
        incl.count += n;
      }
    }
    if ((tid & 31) == 31) {
      sh->part_scan[tid >> 5] = incl.mass;
      sh->part_scan_n[tid >> 5] = incl.count;
    }
    __syncthreads();
    Tally total{0, 0, 0};
    for (int w = 0; w < nt / 32; ++w) {
      if (w == (tid >> 5)) {
        incl.mass += total.mass;
        incl.count += total.count;
      }
      total.mass += sh->part_scan[w];
      total.count += sh->part_scan_n[w];
    }
    if (tid < c.ctas) {
      st_peer(&sh->parts[c.rank].mass, tid, total.mass);
      st_peer(&sh->parts[c.rank].count, tid, total.count);
    }
    row_sync();
    Tally base = above;
    for (int r = 0; r < c.rank; ++r) {
      base.mass += sh->parts[r].mass;
      base.count += sh->parts[r].count;
    }
    // The thread whose bins hold the place where the run reaches `want`.
    const unsigned long long before =
        kByMass ? base.mass + incl.mass - mine.mass : base.count + incl.count - mine.count;
    const unsigned long long after =
        kByMass ? base.mass + incl.mass : static_cast<unsigned long long>(base.count) + incl.count;
    if (before < want && want <= after) {
      Tally run{base.mass + incl.mass - mine.mass, base.count + incl.count - mine.count, 0};
      for (int j = 0; j < per; ++j) {
        const int b = kBins - 1 - (c.rank * share + tid * per + j);
        Tally t{0, 0, 0};
        for (int r = 0; r < c.ctas; ++r) {
          t.count += ld_peer(&sh->count[b], r);
          if (kByMass) t.mass += ld_peer(&sh->mass[b], r);
        }
        const unsigned long long reach =
            kByMass ? run.mass + t.mass : static_cast<unsigned long long>(run.count) + t.count;
        if (reach >= want) {
          for (int r = 0; r < c.ctas; ++r) {
            st_peer(&sh->found.mass, r, run.mass);
            st_peer(&sh->found.count, r, run.count);
            st_peer(&sh->found_bin, r, static_cast<uint32_t>(b));
            st_peer(&sh->found_at.mass, r, t.mass);
            st_peer(&sh->found_at.count, r, t.count);
          }
          break;
        }
        run.mass += t.mass;
        run.count += t.count;
      }
    }
    row_sync();
    above = sh->found;
    const uint32_t b = sh->found_bin;
    const Tally at = sh->found_at;  // written again two cluster_syncs from here
    const uint32_t from = lo + (b << shift);
    if (shift == 0) return Cut{from, above, at};
    hi = min(hi, from + ((1u << shift) - 1u));
    lo = from;
  }
}

// The element at which the running weight in index order first exceeds `drawn`:
// its index, in the one thread of the cluster that finds it; -1 in the others.
// weight(i) is the weight of element i of the row (0: not taking part), parts
// the weight of each CTA's slice (cluster_exchange).  Each thread of the CTA
// that holds the place adds up a run of its own; an odd number of elements, so
// that the threads' reads fall into different banks.
template <typename T, typename Weight>
__device__ __forceinline__ int find_index(const RowCta& c, const Slice<T>& s,
                                          const unsigned long long* parts,
                                          unsigned long long drawn, Weight&& weight) {
  unsigned long long base = 0;
  int owner = 0;
  for (; owner < c.ctas - 1 && drawn >= base + parts[owner]; ++owner) base += parts[owner];
  if (owner != c.rank) return -1;
  const int tid = threadIdx.x, nt = blockDim.x;
  const int n = s.hi - s.lo, per = ((n + nt - 1) / nt) | 1;
  const int a = min(n, tid * per), b = min(n, a + per);
  unsigned long long own = 0;
  for (int i = a; i < b; ++i) own += weight(s.lo + i);
  unsigned long long incl = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long m = __shfl_up_sync(0xffffffffu, incl, o);
    if ((tid & 31) >= o) incl += m;
  }
  __syncthreads();  // wred is free
  if ((tid & 31) == 31) c.sh->wred[0][tid >> 5] = incl;
  __syncthreads();
  for (int w = 0; w < (tid >> 5); ++w) incl += c.sh->wred[0][w];
  unsigned long long run = base + incl - own;
  if (drawn < run || drawn >= run + own) return -1;
  for (int i = a; i < b; ++i) {
    run += weight(s.lo + i);
    if (drawn < run) return s.lo + i;
  }
  return -1;
}

// The index that one thread of the cluster found (>= 0 there), in every thread.
__device__ __forceinline__ int tell_index(const RowCta& c, int found) {
  if (found >= 0)
    for (int r = 0; r < c.ctas; ++r)
      st_peer(reinterpret_cast<const uint32_t*>(&c.sh->told), r, static_cast<uint32_t>(found));
  row_sync();
  return c.sh->told;
}

// ------------------------------------------------------------- candidates --

// A key with at least `count` elements of this CTA's slice at or above it, near
// the largest such: the count-th largest of the threads' maxima (each stands for
// an element), its lower 16 bits cleared in 32-bit keys.  0 where the CTA has
// fewer threads than that.  All threads call it.
template <typename T>
__device__ __forceinline__ uint32_t local_floor(float thread_max, int count) {
  constexpr int kDrop = Row<T>::kKeyBits - 16;
  const uint32_t key = key_of<T>(thread_max) >> kDrop;
  uint32_t found = 0;
#pragma unroll 1
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t t = found | (1u << bit);
    if (__syncthreads_count(key >= t) >= count) found = t;
  }
  return found << kDrop;
}

// Order of candidates: falling key, then rising index.
__device__ __forceinline__ unsigned long long candidate(uint32_t key, int index) {
  return (static_cast<unsigned long long>(~key) << 32) | static_cast<uint32_t>(index);
}
__device__ __forceinline__ uint32_t candidate_key(unsigned long long x) {
  return ~static_cast<uint32_t>(x >> 32);
}
__device__ __forceinline__ int candidate_index(unsigned long long x) {
  return static_cast<int>(static_cast<uint32_t>(x));
}

// Appends a candidate to CTA 0's list; past its end they are only counted.
__device__ __forceinline__ void push_candidate(const RowCta& c, uint32_t key, int index) {
  uint32_t at;
  asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], 1;"
               : "=r"(at)
               : "r"(mapa_shared(&c.sh->listed, 0))
               : "memory");
  if (at < kListMax) st_peer(c.sh->list + at, 0, candidate(key, index));
}

// Sorts n (a power of two) 64-bit values in shared memory, rising.
__device__ __forceinline__ void cta_sort(unsigned long long* a, int n) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int q = threadIdx.x; q < n / 2; q += blockDim.x) {
        const int i = ((q & ~(j - 1)) << 1) | (q & (j - 1));
        const unsigned long long x = a[i], y = a[i + j];
        if ((x > y) == ((i & k) == 0)) {
          a[i] = y;
          a[i + j] = x;
        }
      }
      __syncthreads();
    }
}
// ... n of any size, with room up to the next power of two.
__device__ __forceinline__ void cta_sort_any(unsigned long long* a, int n) {
  const int size = n > 1 ? 1 << (32 - __clz(n - 1)) : 1;
  for (int i = n + threadIdx.x; i < size; i += blockDim.x) a[i] = ~0ull;
  __syncthreads();
  cta_sort(a, size);
}

// The sum of the values before this thread's, and of all.
__device__ __forceinline__ unsigned long long cta_scan(const RowCta& c, unsigned long long v,
                                                       unsigned long long& whole) {
  unsigned long long incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long m = __shfl_up_sync(0xffffffffu, incl, o);
    if ((threadIdx.x & 31) >= o) incl += m;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 31) c.sh->wred[0][threadIdx.x >> 5] = incl;
  __syncthreads();
  unsigned long long before = incl - v;
  whole = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {
    if (w < static_cast<int>(threadIdx.x >> 5)) before += c.sh->wred[0][w];
    whole += c.sh->wred[0][w];
  }
  return before;
}

// The cluster that reads a row: as few CTAs as keep a slice within
// kSliceTarget, more while the grid leaves SMs idle and slices stay long.
__host__ __forceinline__ int row_ctas(int M, int V, int elem, int sms) {
  constexpr size_t kSliceTarget = 40 * 1024;
  int c = 1;
  while (c < kRowMaxCluster && row_slice_bytes(V, c, elem) > kSliceTarget) c *= 2;
  while (c < kRowMaxCluster && static_cast<long long>(M) * c * 2 <= sms && V / c > 4096) c *= 2;
  return c;
}

// Threads of a CTA: about 8 elements for each, whole warps.
__host__ __forceinline__ int row_threads(int V, int ctas) {
  const int n = (row_chunk(V, ctas) + 7) / 8;
  return n < 128 ? 128 : n > kRowMaxThreads ? kRowMaxThreads : (n + 31) / 32 * 32;
}

}  // namespace cai
