// What the operators on rows of vocabulary logits share.  HBM is read once and no
// call needs a workspace, in two forms of the same kernels:
//
//   Cluster (few rows): a row is cut over the CTAs of one thread-block cluster,
//   each keeps its slice in shared memory for every pass it makes, and the
//   cluster reduces and searches through distributed shared memory.
//   Alone (many rows): one CTA takes a row; passes after the first read it from
//   L2, where the rows in progress fit, and nothing waits for another CTA.
#pragma once

#include <climits>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"

namespace cai {

constexpr int kRowMaxCluster = 8;    // portable cluster size
constexpr int kRowMaxThreads = 512;
constexpr int kAloneShare = 2;       // CTAs of 512 threads alone on an SM
constexpr int kRowMaxWarps = kRowMaxThreads / 32;

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

// The largest of a thread's elements, in parts: each part of a vector has a maximum
// of its own, NaN kept.
template <typename T>
struct Maxima;
template <>
struct Maxima<float> {
  static constexpr int kParts = 2;
  float a, b;
  __device__ __forceinline__ Maxima() : a(-__builtin_huge_valf()), b(a) {}
  // Adds a vector; returns its largest element.
  __device__ __forceinline__ float add(const uint4& v) {
    const float x = max_nan(__uint_as_float(v.x), __uint_as_float(v.y));
    const float y = max_nan(__uint_as_float(v.z), __uint_as_float(v.w));
    a = max_nan(a, x);
    b = max_nan(b, y);
    return max_nan(x, y);
  }
  __device__ __forceinline__ float part(int i) const { return i ? b : a; }
  __device__ __forceinline__ float all() const { return max_nan(a, b); }
};
template <>
struct Maxima<__nv_bfloat16> {
  static constexpr int kParts = 4;
  uint32_t a, b;
  __device__ __forceinline__ Maxima() : a(0xff80ff80u), b(a) {}
  static __device__ __forceinline__ float of(uint32_t r) {
    return max_nan(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u));
  }
  __device__ __forceinline__ float add(const uint4& v) {
    const uint32_t x = max2_nan(v.x, v.y), y = max2_nan(v.z, v.w);
    a = max2_nan(a, x);
    b = max2_nan(b, y);
    return of(max2_nan(x, y));
  }
  __device__ __forceinline__ float part(int i) const {
    const uint32_t r = i & 2 ? b : a;
    return __uint_as_float(i & 1 ? r & 0xffff0000u : r << 16);
  }
  __device__ __forceinline__ float all() const { return of(max2_nan(a, b)); }
};

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

// (No memory clobber: what a loop holds in registers stays there.  Where a row's
// gradient is written in place of its logits, each vector is written by the thread
// that has just read it.)
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// ... of a row that is read again soon, and for the last time.
__device__ __forceinline__ uint4 ld_hint(const uint4* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy));
  return v;
}

// The slice of a row that this CTA works on: elements [lo, hi).  It is seen as
// 16-byte vectors of global memory; what the first or last of them holds besides
// the slice is taken as -inf and never read.  Vector v covers the elements
// lo - skip + v kVec ...; vectors outside [first, last) are such ends and lie in
// edge[0] (v = 0) or edge[1].  Once loaded, vector v lies in kept[v] for v < keep;
// kKeep: every one, the ends too.
template <typename T, bool kKeep>
struct Slice {
  static constexpr int kVec = Row<T>::kVec;
  static constexpr bool kKept = kKeep;  // ends are vectors like the others then
  const T* row;
  const uint4* src;
  uint4* kept;
  uint4* edge;
  int n_vec, first, last;
  int keep;
  int lo, hi;
  int skip;

  __device__ __forceinline__ Slice(const T* row_, int lo_, int hi_, uint4* kept_, int room, uint4* edge_)
      : row(row_), kept(kept_), edge(edge_), lo(lo_), hi(hi_) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + lo);
    src = reinterpret_cast<const uint4*>(at & ~static_cast<uintptr_t>(15));
    skip = static_cast<int>((at & 15) / sizeof(T));
    const int span = skip + hi - lo;
    n_vec = hi > lo ? (span + kVec - 1) / kVec : 0;
    first = skip ? 1 : 0;
    last = max(first, span / kVec);
    if (n_vec == 0) first = last = 0;
    keep = kKeep ? n_vec : min(room, last);
  }
  __device__ __forceinline__ int index(int v) const { return lo - skip + v * kVec; }
  __device__ __forceinline__ bool holds(int i) const { return i >= lo && i < hi; }
  // The end that thread `tid` looks after (-1: none): the first two threads do.
  __device__ __forceinline__ int end_of(int tid) const {
    return tid == 0 ? (first > 0 && n_vec > 0 ? 0 : -1) : tid == 1 && last < n_vec ? n_vec - 1 : -1;
  }
  // The value of an element, once the slice is loaded.
  __device__ __forceinline__ float value(int i) const {
    return Row<T>::to_float(kKeep ? reinterpret_cast<const T*>(kept)[i - index(0)] : row[i]);
  }
  // Any vector from where the slice lies now.
  __device__ __forceinline__ uint4 get(int v) const {
    if (kKeep || (v >= first && v < keep)) return kept[v];
    if (v >= first && v < last) return ld_stream(src + v);
    return edge[v != 0 || first == 0];
  }
};

// Calls f(v, vector) for the vectors v = from, from + step, ... below `end`, from
// memory at `src` (shared or global), kFlight loads at a time.  The last round is
// like the others, with fewer loads: one by one its vectors would wait for memory
// as often as all the rounds before.
template <int kFlight, bool kShared, bool kHint = false, typename F>
__device__ __forceinline__ void for_vectors(const uint4* src, int from, int end, int step, F&& f,
                                            uint64_t policy = 0) {
#pragma unroll 1
  for (int v = from; v < end; v += kFlight * step) {
    uint4 r[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (v + j * step < end) {
        const uint4* p = src + v + j * step;
        r[j] = kShared ? *p : kHint ? ld_hint(p, policy) : ld_stream(p);
      }
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (v + j * step < end) f(v + j * step, r[j]);
  }
}

// ... of a loaded slice, from where they lie; its ends are left out (!kKeep).
template <int kFlight, bool kLast = false, typename T, bool kKeep, typename F>
__device__ __forceinline__ void for_body(const Slice<T, kKeep>& s, int from, int end, int step, F&& f) {
  if (kKeep) {
    for_vectors<kFlight, true>(s.kept, from, end, step, f);
    return;
  }
  if (from < s.first) from += step;
  for_vectors<kFlight, true>(s.kept, from, min(end, s.keep), step, f);
  if (from < s.keep) from += (s.keep - from + step - 1) / step * step;
  if (kLast)
    for_vectors<kFlight, false, true>(s.src, from, min(end, s.last), step, f, policy_evict_first());
  else
    for_vectors<kFlight, false>(s.src, from, min(end, s.last), step, f);
}

// Calls f(v, vector) for every vector of the slice, each thread its share.  kLast:
// nothing reads the row again.
template <int kFlight, bool kLast = false, typename T, bool kKeep, typename F>
__device__ __forceinline__ void for_slice(const Slice<T, kKeep>& s, F&& f) {
  const int tid = threadIdx.x, step = static_cast<int>(blockDim.x);
  for_body<kFlight, kLast>(s, tid, s.n_vec, step, f);
  const int end = kKeep ? -1 : s.end_of(tid);
  if (end >= 0) f(end, s.get(end));
}

// The first pass over the vectors [a, b) but the ends, from global memory; keeps
// what there is room for.
template <int kFlight, typename T, bool kKeep, typename F>
__device__ __forceinline__ void load_part(const Slice<T, kKeep>& s, int a, int b, F&& f) {
  const int step = static_cast<int>(blockDim.x);
  int from = threadIdx.x;
  a = max(a, s.first);
  if (from < a) from += (a - from + step - 1) / step * step;
  const auto see = [&](int v, const uint4& r) {
    if (kKeep || v < s.keep) s.kept[v] = r;
    f(v, r);
  };
  if (kKeep)
    for_vectors<kFlight, false>(s.src, from, min(b, s.last), step, see);
  else
    for_vectors<kFlight, false, true>(s.src, from, min(b, s.last), step, see, policy_evict_last());
}

// ... and over the ends, which it builds.
template <typename T, bool kKeep, typename F>
__device__ __forceinline__ void load_ends(const Slice<T, kKeep>& s, F&& f) {
  const int end = s.end_of(threadIdx.x);
  if (end < 0) return;
  uint4 r;
  T* d = reinterpret_cast<T*>(&r);
#pragma unroll
  for (int e = 0; e < Row<T>::kVec; ++e) {
    const int i = s.index(end) + e;
    d[e] = s.holds(i) ? s.row[i] : Row<T>::neg_inf();
  }
  if (kKeep)
    s.kept[end] = r;
  else
    s.edge[end != 0 || s.first == 0] = r;
  f(end, r);
}

template <int kFlight, typename T, bool kKeep, typename F>
__device__ __forceinline__ void load_slice(const Slice<T, kKeep>& s, F&& f) {
  load_part<kFlight>(s, 0, s.n_vec, f);
  load_ends(s, f);
}

// Elements per CTA of a row of V over `ctas`: a multiple of 64.
__host__ __device__ __forceinline__ int row_chunk(int V, int ctas) {
  return ((V + ctas - 1) / ctas + 63) / 64 * 64;
}
// Shared memory of a slice, with room for the shifted start.
__host__ __device__ __forceinline__ size_t row_slice_bytes(int V, int ctas, int elem) {
  return static_cast<size_t>(row_chunk(V, ctas)) * elem + 32;
}

template <typename T, bool kKeep>
__device__ __forceinline__ Slice<T, kKeep> row_slice(const T* row, int V, int rank, int ctas,
                                                     void* smem, int room, uint4* edge) {
  const int chunk = kKeep ? row_chunk(V, ctas) : V;
  const int lo = min(V, rank * chunk);
  return Slice<T, kKeep>(row, lo, min(V, lo + chunk), static_cast<uint4*>(smem), room, edge);
}

// ------------------------------------------------------ reductions, search --

constexpr int kBins = 1024;
constexpr int kListMax = 2048;  // candidates that one CTA finishes alone
constexpr int kSums = 3;        // values of an exchange

// Shared memory of a CTA beside its slice.
struct RowShared {
  unsigned long long wred[kSums][kRowMaxWarps];          // values per warp
  unsigned long long slots[4][kSums][kRowMaxCluster];    // values per CTA, written by the peers
  unsigned long long parts[kRowMaxCluster];
  struct {                // the bin a level found (search_level)
    unsigned long long before;
    int bin;
    uint32_t count;
  } found;
  uint32_t told[2];       // what one thread found, for all (tell)
  unsigned long long once;  // what one warp worked out, for the CTA (cta_once)
  uint4 edge[2];          // the slice's ends
  uint32_t listed;        // candidates pushed so far (in CTA 0)
  uint32_t noted;         // vectors noted so far
  uint32_t note[kListMax];  // vectors with candidates
  union {
    uint32_t count[kBins];               // search_level
    unsigned long long list[kListMax];  // candidates (in CTA 0)
  };
};

// A CTA's place in the cluster that works on its row; kCluster false: there is no
// other.
template <bool kCluster>
struct RowCta {
  RowShared* sh;
  int rank_, ctas_;
  int turn = 0;  // which slots the next exchange uses

  __device__ __forceinline__ RowCta(RowShared* s, int ctas)
      : sh(s), rank_(kCluster ? static_cast<int>(cluster_ctarank()) : 0), ctas_(ctas) {}
  __device__ __forceinline__ int rank() const { return kCluster ? rank_ : 0; }
  __device__ __forceinline__ int ctas() const { return kCluster ? ctas_ : 1; }

  // Peers' shared memory may be written once every CTA of the cluster has begun:
  // begin at the top of a kernel, begun before the first such write (and before
  // any early return).
  __device__ __forceinline__ static void begin() {
    if (kCluster) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  }
  __device__ __forceinline__ void begun() const {
    if (!kCluster) return;
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  // All threads of the row.  Warps may arrive from loops that their lanes left at
  // different times.
  __device__ __forceinline__ void sync() const {
    if (kCluster) {
      __syncwarp();
      cluster_sync();
    } else {
      __syncthreads();
    }
  }
  // Writes into, or reads from, `p`'s place in the shared memory of CTA `rank`.
  __device__ __forceinline__ void store(unsigned long long* p, int rank, unsigned long long v) const {
    if (kCluster)
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_shared(p, rank)), "l"(v) : "memory");
    else
      *p = v;
  }
  __device__ __forceinline__ void store(uint32_t* p, int rank, uint32_t v) const {
    if (kCluster)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_shared(p, rank)), "r"(v) : "memory");
    else
      *p = v;
  }
  __device__ __forceinline__ unsigned long long load(const unsigned long long* p, int rank) const {
    if (!kCluster) return *p;
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(mapa_shared(p, rank)) : "memory");
    return v;
  }
  __device__ __forceinline__ uint32_t load(const uint32_t* p, int rank) const {
    if (!kCluster) return *p;
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(p, rank)) : "memory");
    return v;
  }
  __device__ __forceinline__ uint32_t next(uint32_t* p, int rank) const {  // p++ there
    if (!kCluster) return atomicAdd(p, 1u);
    uint32_t v;
    asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], 1;"
                 : "=r"(v)
                 : "r"(mapa_shared(p, rank))
                 : "memory");
    return v;
  }
};

template <typename Op>
__device__ __forceinline__ unsigned long long warp_reduce(unsigned long long v, Op op) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Reduces one value per thread over the CTA, the result in every thread.  All
// threads call it; wred is free again after the next barrier.
template <typename Op>
__device__ __forceinline__ unsigned long long cta_reduce(RowShared* sh, unsigned long long v, Op op,
                                                         int which = 0) {
  v = warp_reduce(v, op);
  const int lane = threadIdx.x & 31, n = blockDim.x >> 5;
  if (lane == 0) sh->wred[which][threadIdx.x >> 5] = v;
  __syncthreads();
  // Lanes repeat the warps' values: n is a power of two here.
  v = sh->wred[which][lane & (n - 1)];
#pragma unroll 1
  for (int o = n >> 1; o >= 1; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
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
#pragma unroll 1
    for (int i = 0; i < ctas; ++i) r += of(which)[i];
    return r;
  }
};
template <int kN, typename C>
__device__ __forceinline__ Parts cluster_exchange(C& c, const unsigned long long (&v)[kN]) {
  unsigned long long* s = &c.sh->slots[c.turn & 3][0][0];
  c.turn++;
  if (static_cast<int>(threadIdx.x) < c.ctas()) {
#pragma unroll
    for (int i = 0; i < kN; ++i) c.store(s + i * kRowMaxCluster + c.rank(), threadIdx.x, v[i]);
  }
  c.sync();
  return Parts{s};
}

struct AddOp {
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return a + b;
  }
};
// The sums of up to three values per thread, CTA by CTA, to all.
template <int kN, typename C>
__device__ __forceinline__ Parts exchange_sums(C& c, const unsigned long long (&v)[kN]) {
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
    r[i] = c.sh->wred[i][threadIdx.x & (n - 1)];
#pragma unroll 1
    for (int o = n >> 1; o >= 1; o >>= 1) r[i] += __shfl_xor_sync(0xffffffffu, r[i], o);
  }
  return cluster_exchange(c, r);
}

__device__ __forceinline__ unsigned long long warp_scan(unsigned long long v) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long m = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += m;
  }
  return v;
}

// The sum of the values before this thread's, and of all.
__device__ __forceinline__ unsigned long long cta_scan(RowShared* sh, unsigned long long v,
                                                       unsigned long long& whole) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockDim.x >> 5;
  const unsigned long long incl = warp_scan(v);
  __syncthreads();
  if (lane == 31) sh->wred[0][warp] = incl;
  __syncthreads();
  const unsigned long long w = warp_scan(lane < n ? sh->wred[0][lane] : 0);
  whole = __shfl_sync(0xffffffffu, w, 31);
  const unsigned long long before = __shfl_sync(0xffffffffu, w, (warp - 1) & 31);
  return (warp ? before : 0) + incl - v;
}

// Where a falling run over the elements of the row first reaches a count: between
// the keys lo and hi, with how many lie above and how many there.
struct Cut {
  uint32_t lo, hi;
  uint32_t above, at;
};

// One level of a search from the largest value down: count(f) calls f(bin) for
// the elements that take part, value(bin, n) is what n elements of a bin add to
// the run, which starts at `run`.  Returns the bin in which it reaches `want` (-1:
// in none), and the run before it and the elements in it.  All threads of all
// CTAs call it.
struct Level {
  int bin;
  unsigned long long before;
  uint32_t count;
};
template <typename C, typename Count, typename Value>
__device__ __forceinline__ Level search_level(C& c, unsigned long long run, unsigned long long want,
                                              Count&& count, Value&& value) {
  RowShared* sh = c.sh;
  const int tid = threadIdx.x, nt = blockDim.x;
#pragma unroll 1
  for (int i = tid; i < kBins; i += nt) sh->count[i] = 0;
  if (tid == 0) sh->found.bin = -1;
  __syncthreads();
  count([&](int b) { atomicAdd(&sh->count[b], 1u); });
  c.sync();
  // Every CTA sums its share of the bins over the cluster; bins fall with the
  // thread index so that a rising scan runs from the largest values down.
  const int share = kBins / c.ctas();
  const int per = (share + nt - 1) / nt;  // bins of a thread
  const auto bin_of = [&](int j) { return kBins - 1 - (c.rank() * share + tid * per + j); };
  const auto sum_bin = [&](int b) {
    uint32_t n = 0;
#pragma unroll 1
    for (int r = 0; r < c.ctas(); ++r) n += c.load(&sh->count[b], r);
    return n;
  };
  unsigned long long mine = 0, total;
#pragma unroll 1
  for (int j = 0; j < per && tid * per + j < share; ++j) mine += value(bin_of(j), sum_bin(bin_of(j)));
  const unsigned long long before = cta_scan(sh, mine, total);
  if (tid < c.ctas()) c.store(&sh->parts[c.rank()], tid, total);
  c.sync();
#pragma unroll 1
  for (int r = 0; r < c.rank(); ++r) run += sh->parts[r];
  run += before;
  // The thread whose bins hold the place where the run reaches `want`.
  if (run < want && want <= run + mine) {
#pragma unroll 1
    for (int j = 0; j < per; ++j) {
      const int b = bin_of(j);
      const uint32_t n = sum_bin(b);
      const unsigned long long v = value(b, n);
      if (run + v >= want) {
#pragma unroll 1
        for (int r = 0; r < c.ctas(); ++r) {
          c.store(&sh->found.before, r, run);
          c.store(reinterpret_cast<uint32_t*>(&sh->found.bin), r, static_cast<uint32_t>(b));
          c.store(&sh->found.count, r, n);
        }
        break;
      }
      run += v;
    }
  }
  c.sync();
  const Level l{sh->found.bin, sh->found.before, sh->found.count};
  __syncthreads();  // read before the next level clears it
  return l;
}

// Radix search for the `want`-th element of the row from the largest down, kBins
// parts of the remaining key range at a time, until it holds at most `enough`
// elements or one key.  visit(f) calls f(key) for every element.
template <typename T, typename C, typename Visit>
__device__ __forceinline__ Cut find_cut(C& c, uint32_t top, uint32_t want, uint32_t enough, Visit&& visit) {
  uint32_t lo = 0, hi = top, above = 0;  // the key is in [lo, hi]
#pragma unroll 1
  for (;;) {
    const uint32_t range = hi - lo;
    const int bits = 32 - __clz(range);  // 0 for one key
    const int shift = bits > 10 ? bits - 10 : 0;
    const Level l = search_level(
        c, above, want,
        [&](auto&& f) {
          visit([&](uint32_t key) {
            if (key - lo <= range) f(static_cast<int>((key - lo) >> shift));
          });
        },
        [](int, uint32_t n) -> unsigned long long { return n; });
    above = static_cast<uint32_t>(l.before);
    const uint32_t from = lo + (static_cast<uint32_t>(max(l.bin, 0)) << shift);
    hi = min(hi, from + ((1u << shift) - 1u));
    lo = from;
    if (shift == 0 || l.count <= enough) return Cut{lo, hi, above, l.count};
  }
}

// ------------------------------------------------------------------ weights --

// A token's weight is a share e in [0, 1] in units of 2^-40, rounded to a whole
// number: sums of weights are exact, whatever their order.
constexpr float kWeightUnit = 1099511627776.0f;  // 2^40
constexpr float kOneUnit = 1.0f / kWeightUnit;   // the share whose weight is 1

// In 32-bit pieces, a few instructions an element: e + 1 rounds e to units of
// 2^-23 and holds them in the low bits; what that leaves is exact, at most 2^-24,
// and is rounded to units of 2^-40 in the low bits of a number near 1.5 2^23.
constexpr uint32_t kOneBits = 0x3f800000u;    // 1.0f
constexpr uint32_t kMagicBits = 0x4b400000u;  // 1.5 * 2^23

__device__ __forceinline__ unsigned long long weight_of(float e) {
  const float h = __fadd_rn(e, 1.0f);
  const float l = __fmaf_rn(__fsub_rn(e, __fsub_rn(h, 1.0f)), kWeightUnit, 12582912.0f);
  return (static_cast<unsigned long long>(__float_as_uint(h) - kOneBits) << 17) +
         static_cast<long long>(static_cast<int32_t>(__float_as_uint(l) - kMagicBits));
}

// The sum of up to 1022 elements' weights in a thread (a row of 2^18 gives 512 and
// its ends to each of 512 threads).  A weight's high part is at most 2^23, so each
// element of a pair has a sum of its own.
struct WeightSum {
  uint32_t high0 = 0, high1 = 0, low = 0;
  __device__ __forceinline__ void add(float e0, float e1) {
    const float2 e = make_float2(e0, e1), one = make_float2(1.0f, 1.0f);
    const float2 h = __fadd2_rn(e, one);
    const float2 r = __fadd2_rn(e, __fadd2_rn(one, make_float2(-h.x, -h.y)));
    const float2 l = __ffma2_rn(r, make_float2(kWeightUnit, kWeightUnit),
                                make_float2(12582912.0f, 12582912.0f));
    high0 += __float_as_uint(h.x);
    high1 += __float_as_uint(h.y);
    low += __float_as_uint(l.x) + __float_as_uint(l.y);
  }
  // After n elements, an even number.
  __device__ __forceinline__ unsigned long long sum(uint32_t n) const {
    const long long lo = static_cast<int32_t>(low - n * kMagicBits);
    const uint32_t ones = n / 2 * kOneBits;
    return ((static_cast<unsigned long long>(high0 - ones) + (high1 - ones)) << 17) + lo;
  }
};

// f() worked out by one warp for the CTA: 64-bit floating point is slow enough for
// sixteen warps to queue for it.
template <typename F>
__device__ __forceinline__ unsigned long long cta_once(RowShared* sh, F&& f) {
  __syncthreads();
  if (threadIdx.x < 32) {
    const unsigned long long v = f();
    if (threadIdx.x == 0) sh->once = v;
  }
  __syncthreads();
  return sh->once;
}

// The element at which the running weight in index order first exceeds a number
// drawn(whole): its index, in the one thread of the row that finds it; -1 in the
// others.  share(i, z0, z1) are those of elements i and i + 1 of values z0, z1 (0:
// not taking part; also asked of what the ends hold besides the slice).  `whole`
// and `found` receive the whole weight and the element's.  All threads call it.
// Each warp adds up a run of vectors; the run that holds the place is then cut
// over the CTA's threads.
template <typename T, typename C, typename S, typename Share, typename Drawn>
__device__ __noinline__ int find_index(C& c, const S s, const Share share, const Drawn drawn_of,
                                       unsigned long long& whole, unsigned long long& found) {
  constexpr int kVec = Row<T>::kVec;
  constexpr bool kKept = S::kKept;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int per = (s.n_vec + warps - 1) / warps;
  unsigned long long* wmass = c.sh->wred[kSums - 1];
  unsigned long long run = 0, drawn = 0;
  // The thread's vectors: of its warp's run, then of the run that holds the place.
  int v = min(s.n_vec, warp * per) + lane, end = min(s.n_vec, warp * per + per), step = 32, first = v;
#pragma unroll 1
  for (int turn = 0;; ++turn) {
    WeightSum sum;
    uint32_t n = 0;
    const auto add = [&](int u, const uint4& r) {
      float z[kVec];
      Row<T>::unpack(r, z);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const float2 w = share(s.index(u) + e, z[e], z[e + 1]);
        sum.add(w.x, w.y);
      }
      n += kVec;
    };
    for_body<4>(s, v, end, step, add);
    // The ends, where they are among this thread's vectors.
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      const int u = s.end_of(k);
      if (!kKept && u >= v && u < end && (u - v) % step == 0) add(u, s.get(u));
    }
    unsigned long long own = sum.sum(n);
    if (turn == 0) {
      own = warp_reduce(own, AddOp());
      if (lane == 0) wmass[warp] = own;
      __syncthreads();
      unsigned long long cta[1] = {0};
#pragma unroll 1
      for (int w = 0; w < warps; ++w) cta[0] += wmass[w];
      const unsigned long long* parts = cluster_exchange(c, cta).of(0);
      whole = 0;
#pragma unroll 1
      for (int q = 0; q < c.ctas(); ++q) {
        if (q == c.rank()) run = whole;
        whole += parts[q];
      }
      drawn = cta_once(c.sh, [&]() { return drawn_of(whole); });
      if (drawn < run || drawn >= run + cta[0]) return -1;  // the same in the whole CTA
      int hold = 0;
#pragma unroll 1
      while (hold < warps - 1 && drawn >= run + wmass[hold]) run += wmass[hold++];
      // Each thread a part of that warp's run.
      const int a = min(s.n_vec, hold * per), b = min(s.n_vec, a + per);
      const int each = (b - a + static_cast<int>(blockDim.x) - 1) / static_cast<int>(blockDim.x);
      first = v = min(b, a + static_cast<int>(threadIdx.x) * each);
      end = min(b, v + each);
      step = 1;
      continue;
    }
    unsigned long long all;
    run += cta_scan(c.sh, own, all);
    if (drawn < run || drawn >= run + own) return -1;
    break;
  }
#pragma unroll 1
  for (int i = max(s.lo, s.index(first)); i < min(s.hi, s.index(end)); ++i) {
    const float z = s.value(i);
    const unsigned long long w = weight_of(share(i, z, z).x);
    run += w;
    if (drawn < run) {
      found = w;
      return i;
    }
  }
  return -1;
}

// Two words that one thread of the row has (`mine`), in every thread.
struct Told {
  uint32_t a, b;
};
template <typename C>
__device__ __forceinline__ Told tell(const C& c, bool mine, uint32_t a, uint32_t b) {
  if (mine)
#pragma unroll 1
    for (int r = 0; r < c.ctas(); ++r) {
      c.store(&c.sh->told[0], r, a);
      c.store(&c.sh->told[1], r, b);
    }
  c.sync();
  return Told{c.sh->told[0], c.sh->told[1]};
}

// ------------------------------------------------------------- candidates --

// The count-th largest of kN 16-bit keys of each lane of a warp; 0 where count is
// above their number.
template <int kN>
__device__ __forceinline__ uint32_t warp_select(const uint32_t (&key)[kN], int count) {
  uint32_t found = 0;
#pragma unroll(kN == 1 ? 16 : 1)
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t t = found | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) n += __popc(__ballot_sync(0xffffffffu, key[i] >= t));
    if (n >= count) found = t;
  }
  return found;
}
// A key with at least `count` elements of this warp's at or above it (0: none is
// known), its lower 16 bits cleared in 32-bit keys: the count-th largest of the
// lanes' maxima, or of their parts' where that lies below the middle of the lanes
// (2048 rows of 4000 bf16, K = 256: the 32nd of 32 250 us, of 128 80; 2000 rows of
// 126464, K = 128: the 8th of 32 177 us, of 128 184).
template <typename T>
__device__ __forceinline__ uint32_t warp_floor(const Maxima<T>& m, int count) {
  constexpr int kDrop = Row<T>::kKeyBits - 16, kParts = Maxima<T>::kParts;
  if (count <= 16) {
    const uint32_t key[1] = {key_of<T>(m.all()) >> kDrop};
    return warp_select(key, count) << kDrop;
  }
  uint32_t key[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) key[i] = key_of<T>(m.part(i)) >> kDrop;
  return warp_select(key, count) << kDrop;
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
template <typename C>
__device__ __forceinline__ void push_candidate(const C& c, uint32_t key, int index) {
  const uint32_t at = c.next(&c.sh->listed, 0);
  if (at < kListMax) c.store(c.sh->list + at, 0, candidate(key, index));
}

// Sorts the first n of 64-bit values in shared memory, rising; no two are alike.
// Returns where they lie then: in `a` (kListMax values of room) or further on in
// it.  Up to half of the room: every warp sorts runs of 32 by shuffles, then each
// value counts the smaller ones of every run by halving, which is its place; three
// barriers (256 values: a network through shared memory took 5.0 us).  More: that
// network, where a warp's 32 pairs of a step with j <= 32 are its own 64 values in
// the step before and after, so only the wider steps wait for other warps.
__device__ __noinline__ unsigned long long* cta_sort(unsigned long long* a, int n) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31;
  __syncthreads();
  if (n <= kListMax / 2) {
    const int runs = (n + 31) / 32;
#pragma unroll 1
    for (int r = tid >> 5; r < runs; r += nt >> 5) {
      const int i = 32 * r + lane;
      unsigned long long x = i < n ? a[i] : ~0ull;
#pragma unroll
      for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
          const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, j);
          if ((x < y) != (((lane & j) == 0) == ((lane & k) == 0))) x = y;
        }
      a[i] = x;  // up to the end of the run
    }
    __syncthreads();
    unsigned long long* out = a + kListMax / 2;
#pragma unroll 1
    for (int i = tid; i < n; i += nt) {
      // (a run's own values are counted like the others: those before i)
      const unsigned long long x = a[i];
      int at = 0;
#pragma unroll 4
      for (int r = 0; r < runs; ++r) {
        const unsigned long long* run = a + 32 * r;
        int c = 0;
#pragma unroll
        for (int h = 16; h > 0; h >>= 1) c += run[c + h - 1] < x ? h : 0;
        at += c + (run[c] < x ? 1 : 0);
      }
      out[at] = x;
    }
    __syncthreads();
    return out;
  }
  int size = kListMax;
  while (size / 2 >= n) size >>= 1;
#pragma unroll 1
  for (int i = n + tid; i < size; i += nt) a[i] = ~0ull;
  int last = 64;  // the step before; before the first everything is waited for
#pragma unroll 1
  for (int k = 2; k <= size; k <<= 1)
#pragma unroll 1
    for (int j = k >> 1; j > 0; j >>= 1) {
      if (j > 32 || last > 32)
        __syncthreads();
      else
        __syncwarp();
      last = j;
#pragma unroll 1
      for (int q = tid; q < size / 2; q += nt) {
        const int i = ((q & ~(j - 1)) << 1) | (q & (j - 1));
        const unsigned long long x = a[i], y = a[i + j];
        if ((x > y) == ((i & k) == 0)) {
          a[i] = y;
          a[i + j] = x;
        }
      }
    }
  __syncthreads();
  return a;
}

// How a call's rows are worked on: ctas 0 stands for the form in which a CTA takes a
// row alone, and keeps `room` vectors of it in shared memory.
struct RowPlan {
  int ctas, threads;
  int room;
  size_t smem;  // dynamic
};
// `extra` bytes beside a slice, `limit` the dynamic shared memory there is for one
// CTA on an SM beside its fixed_smem.
__host__ __forceinline__ RowPlan row_plan(int M, int V, int elem, int sms, size_t limit,
                                          size_t fixed_smem, size_t (*extra)(int)) {
  // A cluster: as few CTAs as keep a slice within 84 KiB, two to an SM (64 rows of
  // 152064 bf16, K = 64: 4 CTAs 16.6 us, 8 26.6), up to four while the
  // grid leaves SMs idle and slices stay long; 256 threads, whose reductions and
  // barriers cost less (one row of 126464 bf16, sampled: 4 CTAs of 256 threads
  // 15.4 us, of 512 16.5, 8 of 256 16.4, 8 of 512 22).
  constexpr size_t kSliceTarget = 84 * 1024;
  int c = 1;
  while (c < kRowMaxCluster && row_slice_bytes(V, c, elem) > kSliceTarget) c *= 2;
  while (c < 4 && static_cast<long long>(M) * c * 2 <= sms && V / c > 4096) c *= 2;
  // Clusters that fill the SMs, two CTAs each, once; of more rows each goes to a CTA
  // alone (126464 bf16, K = 64: 64 rows 16.9 us either way, 90 23.8 and 17.0, 152 34
  // and 18, 304 58 and 24; loss and gradient: 64 rows 17 and 23, 90 27 and 23), but
  // half as many again of the longest, which take one CTA long (152064 float32, loss
  // and gradient: 50 rows 31 and 39, 100 47 and 46; K = 64: 25 and 29, 42 and 29).
  if (c == 1 || static_cast<long long>(M) * c <= (c == kRowMaxCluster ? 3ll : 2ll) * sms)
    return RowPlan{c, 256, 0, row_slice_bytes(V, c, elem) + extra(row_chunk(V, c))};
  // Alone, two on an SM: what shared memory that leaves, in whole rounds of the
  // CTA's threads.
  constexpr size_t kReserved = 1024;  // per CTA, by the system
  const size_t whole = (limit + fixed_smem + kReserved) / kAloneShare;
  const size_t taken = kReserved + fixed_smem + extra(V);
  const size_t round = static_cast<size_t>(kRowMaxThreads) * 16;
  const size_t row = (static_cast<size_t>(V) * elem + 32) / round * round;
  size_t keep = (whole > taken ? whole - taken : 0) / round * round;
  if (keep > row) keep = row;
  return RowPlan{0, kRowMaxThreads, static_cast<int>(keep / 16), keep + extra(V)};
}

}  // namespace cai
