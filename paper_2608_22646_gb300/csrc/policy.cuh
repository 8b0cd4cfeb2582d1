// Log-probabilities of drawn tokens, the clipped policy loss on them, and the
// gradients by the logits (cai_token_logp, cai_policy_loss and their backward
// calls).  With m = max z, e_v = 2^((z_v - m) log2(e) / T) and s = sum e:
//   logp = (z_t - m) / T - ln s,   dlogp/dz_v = ([v = t] - e_v / s) / T,
// and every loss of a row is a function of its logp: its gradient by the logits is
// dloss/dlogp times that.  m and s are the row's stats; differences of logits are
// taken before the product, as in the distillation loss.
#pragma once

#include "async_copy.cuh"
#include "row_ops.cuh"
#include "sample.cuh"
#include "softmax.cuh"
#include "vector_parts.cuh"

namespace cai {

struct TokenParams {
  const void* logits;
  long long ld;
  int M, V;
  const int32_t* token;     // [M], outside [0, V): the row takes no part
  float tau;
  double inv_tau;
  bool policy;              // the clipped loss; else log-probabilities alone
  const float* old_logp;    // [M] or null
  const float* advantage;   // [M]
  const float* ref_logp;    // [M] or null
  const float* weight;      // [M] or null
  float low, high, kl;      // the clip's bounds, the KL term's factor
  float* loss;              // [M] (policy)
  float* logp;              // [M]
  float* stats;             // [M, 2]: m and s
  float* slope;             // [M], dloss/dlogp: written by the loss, read by the gradient; or null
  const float* upstream;    // [M], the backward call's gradient; else null
  void* grad;               // [M, ld_grad] or null
  long long ld_grad;
};

// A running maximum of logits and the sum of 2^((z - m) c2) as s + c: c holds what
// rounding took from s.  A row's largest term is 1; what lies below it by 2^24 and more would
// vanish lane by lane, and always from below.
struct RowSum {
  float m, s, c;
};
__device__ __forceinline__ float token_share(float z, float from, float c2) {
  return fast_exp2(__fmul_rn(__fsub_rn(z, from), c2));
}
// a + b, with the rounding error's negative taken by c.
__device__ __forceinline__ float summed(float a, float b, float& c) {
  const float t = __fadd_rn(a, b), d = __fsub_rn(t, a);
  c = __fadd_rn(c, __fadd_rn(__fsub_rn(a, __fsub_rn(t, d)), __fsub_rn(b, d)));
  return t;
}
__device__ __forceinline__ RowSum merged(RowSum a, RowSum b, float c2) {
  const float m = max_nan(a.m, b.m);
  // -inf on both sides: no element yet.
  const float ea = a.m == m ? 1.0f : token_share(a.m, m, c2);
  const float eb = b.m == m ? 1.0f : token_share(b.m, m, c2);
  RowSum r{m, 0.0f, a.c * ea + b.c * eb};
  r.s = summed(a.s * ea, b.s * eb, r.c);
  return r;
}

// The vectors of 16 bytes that lie whole in elements [lo, hi) of a row: [first, last)
// from src; and the elements before and after them.
// (kEdges false: rows of whole vectors.)
template <typename T, bool kEdges = true>
struct Span {
  static constexpr int kVec = Row<T>::kVec;
  const uint4* src;
  int skip, first, last, lo, hi;
  int n_vec;  // with the ends
  __device__ __forceinline__ Span(const T* row, int lo_, int hi_) : lo(lo_), hi(hi_) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + lo);
    src = reinterpret_cast<const uint4*>(kEdges ? at & ~static_cast<uintptr_t>(15) : at);
    skip = kEdges ? static_cast<int>((at & 15) / sizeof(T)) : 0;
    first = skip ? 1 : 0;
    last = (skip + hi - lo) / kVec;
    if (last < first) last = first;  // no whole vector
    n_vec = hi > lo ? (skip + hi - lo + kVec - 1) / kVec : 0;
  }
  __device__ __forceinline__ int index(int v) const { return lo - skip + v * kVec; }
  // Elements outside the vectors: head() of them from lo, and from tail() on.
  __device__ __forceinline__ int tail() const { return last > first ? index(last) : lo; }
  __device__ __forceinline__ int head() const { return last > first ? index(first) - lo : 0; }
  __device__ __forceinline__ int ends() const { return head() + hi - tail(); }
  __device__ __forceinline__ int end(int i) const { return i < head() ? lo + i : tail() + i - head(); }
};

// What becomes of a row beside its sum, known before that.
struct TokenRow {
  float old_logp, advantage, ref_logp, weight;
};

// A row's loss and its derivative by logp, weight included.
__device__ __forceinline__ void policy_terms(const TokenParams& p, const TokenRow& row, float logp, float& loss,
                                             float& by) {
  const float A = row.advantage;
  float ratio = p.old_logp ? expf(logp - row.old_logp) : 1.0f;
  if (!p.old_logp && logp != logp) ratio = logp;  // no softmax, no loss
  if (ratio > 3.4028235e38f) ratio = 3.4028235e38f;
  const float free = ratio * A;
  const float held = (ratio < p.low ? p.low : ratio > p.high ? p.high : ratio) * A;
  const bool clipped = p.old_logp && free > held;
  loss = clipped ? -held : -free;
  by = clipped ? 0.0f : -free;
  if (p.kl != 0.0f) {
    const float d = row.ref_logp - logp;
    float k;  // exp(d) - d - 1
    if (fabsf(d) < 0.25f)  // its series: the difference would lose d's digits
      k = d * d * (0.5f + d * (1.0f / 6 + d * (1.0f / 24 + d * (1.0f / 120 + d * (1.0f / 720 + d * (1.0f / 5040))))));
    else
      k = expm1f(d) - d;
    loss += p.kl * k;
    by -= p.kl * expm1f(d);
  }
  if (p.weight) {
    loss *= row.weight;
    by *= row.weight;
  }
}

// The hardware's 2^x is low by 5.06e-8 of itself on average (x in [-16, 0], and much the
// same in every sixteenth of a binade), which sums over a sequence's tokens would add
// up; and so would roundings that lean one way.  So what is written takes that back
// from the exponentials below the largest, 1, and is rounded once.
constexpr double kExp2Low = 5.06e-8;
__device__ __forceinline__ float token_logp_written(float zt, float m, float s, float rest, double inv_tau) {
  // log(s + rest) with the exponentials below 1 as they would be
  const float more = __fdiv_rn(rest + static_cast<float>(kExp2Low) * fmaxf(s - 1.0f, 0.0f), s);
  return static_cast<float>((static_cast<double>(zt) - m) * inv_tau - logf(s) - more);
}

__device__ __forceinline__ float token_logp_of(float zt, float m, float s, float tau) {
  return __fdiv_rn(zt - m, tau) - logf(s);
}

// ------------------------------------------------------------- rows in turn --

// A cluster of CTAs takes rows in turn, its CTAs a slice of the row each, and logits
// come ahead of the work through a ring of slots in shared memory: asynchronous
// copies of 16 bytes, each into a slot that its own thread reads, so that neither
// loads nor slots need a barrier.  A warp has kBatch times 32 vectors of a batch, side by side;
// a batch is worked on at once and is one group of copies.  Every batch has
// its place and its group, empty ones too: after the first `ring` batches one is asked
// for whenever one is done with, so the number of groups younger than a given batch's
// is known.
//
// Loss and gradient (kGrad): a row's batches stay in the ring from the pass that adds up
// the exponentials to the one that writes the gradient, which frees them.  Else a batch
// is free once it is added.
//
// HBM bounds both: 2048 rows of 126464 bf16, one in eight and one in sixteen without a
// part, loss and gradient in one pass 160 us, of 143 at the copy's rate (two kernels,
// which read the logits twice: 239); the losses alone, all rows, 84, of 76.  (Vectors a CTA's
// threads apart instead of a warp's lanes: 168 and 88.)  Rows that start anywhere: 2000 of 126465
// bf16 188 us and 92, of 149 and 75; with the gradient in another place to its 16 bytes, 248
// (two kernels 290).  What is left is the instructions around 16 bytes and
// the time from a row's sum to its gradient, which the other CTAs of an SM cover in part.
struct TokenPlan {
  int ctas;     // of a cluster
  int threads;
  int batches;  // of a row
  int ring;     // batches; with the gradient, more than a row's; under three rows'
  int clusters;
  int late_turn;  // (a test's form alone: before its sums of this turn a CTA waits past the others' limit)
};

// How rows lie: whole vectors of 16 bytes; anywhere, logits and gradient alike; the gradient
// in another place to its 16 bytes than the logits.
enum TokenEnds { kWhole, kCut, kShifted };

constexpr int kTokenMaxWarps = 8;
constexpr int kBatch = 4;

// What the CTAs of a cluster tell each other of a row, in turn in one of two places: a
// row's is written again for the next but one, which takes every warp's sum of the
// next, which it gives when it has read this one's.
//
// A warp whose wait runs out is deaf from there on: it tells nothing more, since it would
// write over what others have not read, and says so to every CTA of the cluster.  Nobody
// can then hear of a later row: who waits becomes deaf as it learns of it, or in its own
// time.  A deaf warp's rows are NaN, loss, stats and gradient, from the row on that it did
// not hear of; a number that was written came from all sums of its row.
struct TokenShared {
  float4 part[2][kRowMaxCluster * kTokenMaxWarps];  // a warp's sum, of every CTA of the cluster
  TokenRow info[2];
  float zt[2];         // the token's logit, from the CTA that has it
  uint64_t full[2];    // counts the bytes of the above
  TokenRow row[4];     // copied with a row's first batch, each field by a thread that gives it on
  unsigned deaf;       // a warp of the cluster is
};

// Writes 4 or 16 bytes into the same place of another CTA's shared memory and counts them at its
// barrier: no fence, which would wait for the gradient's stores too.
__device__ __forceinline__ void tell(float* dst, uint64_t* bar, int rank, float x) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(mapa_shared(dst, rank)),
               "r"(__float_as_uint(x)), "r"(mapa_shared(bar, rank))
               : "memory");
}
__device__ __forceinline__ void tell(float4* dst, uint64_t* bar, int rank, const RowSum& x) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                   mapa_shared(dst, rank)),
               "r"(__float_as_uint(x.m)), "r"(__float_as_uint(x.s)), "r"(__float_as_uint(x.c)), "r"(0u),
               "r"(mapa_shared(bar, rank))
               : "memory");
}
__device__ __forceinline__ void tell_deaf(unsigned* flag, int rank) {
  asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], 1;" ::"r"(mapa_shared(flag, rank)) : "memory");
}
__device__ __forceinline__ bool any_deaf(const unsigned* flag) {
  uint32_t x;
  asm volatile("ld.relaxed.cluster.shared::cta.u32 %0, [%1];" : "=r"(x) : "r"(smem_addr(flag)) : "memory");
  return x != 0;
}
// Waits for a phase; false after `limit` ns, or where a warp of the cluster is deaf.
__device__ __forceinline__ bool heard(uint64_t* bar, uint32_t parity, const unsigned* flag, uint64_t limit) {
  if (mbar_try_wait_cluster(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait_cluster(bar, parity)) return true;
    if ((it & 63u) == 0u && (any_deaf(flag) || global_timer_ns() - t0 > limit)) return false;
  }
}
__device__ __forceinline__ void pause_ns(uint64_t ns) {
  const uint64_t t0 = global_timer_ns();
  while (global_timer_ns() - t0 < ns) __nanosleep(1000);
}

__device__ __forceinline__ float warp_max_nan(float v) {
  float r;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// The sum over a warp's lanes, in every lane.  (kExact: with what rounding takes.  Loss
// and gradient in one kernel go without until the CTAs' sums meet: 3 % of the time,
// for log-probabilities good to 1.3e-7 and not 6e-8.)
template <bool kExact>
__device__ __forceinline__ RowSum warp_merged(RowSum a, float c2) {
  const float m = warp_max_nan(a.m);
  const float e = a.m == m ? 1.0f : token_share(a.m, m, c2);  // (-inf everywhere: no element, 0)
  RowSum r{m, a.s * e, a.c * e};
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    if (kExact) {
      const float other = __shfl_xor_sync(0xffffffffu, r.c, o);
      r.s = summed(r.s, __shfl_xor_sync(0xffffffffu, r.s, o), r.c);
      r.c += other;
    } else {
      r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
    }
  }
  return r;
}

// The largest logit of a batch, NaN kept.
__device__ __forceinline__ float batch_max(const uint4 (&q)[kBatch], float) {
  float m = vec_max(q[0], -__builtin_huge_valf(), 0.0f);
#pragma unroll
  for (int b = 1; b < kBatch; ++b) m = vec_max(q[b], m, 0.0f);
  return m;
}
__device__ __forceinline__ float batch_max(const uint4 (&q)[kBatch], __nv_bfloat16 t) {
  uint4 m = q[0];
#pragma unroll
  for (int b = 1; b < kBatch; ++b) {
    m.x = max2_nan(m.x, q[b].x);
    m.y = max2_nan(m.y, q[b].y);
    m.z = max2_nan(m.z, q[b].z);
    m.w = max2_nan(m.w, q[b].w);
  }
  return vec_max(m, -__builtin_huge_valf(), t);
}

// A batch's exponentials added to a row's sum.
template <typename T, bool kExact>
__device__ __forceinline__ void add_batch(RowSum& r, const uint4 (&q)[kBatch], float c2) {
  constexpr int kVec = Row<T>::kVec;
  const float top = batch_max(q, T());
  if (!(top <= r.m)) {  // a new maximum, or NaN
    const float e = r.m == -__builtin_huge_valf() ? 0.0f : token_share(r.m, top, c2);
    r.s *= e;
    r.c *= e;
    r.m = top;
  }
  if (r.m == -__builtin_huge_valf()) return;
  float2 e2[2] = {};
#pragma unroll
  for (int b = 0; b < kBatch; ++b) {
    float z[kVec];
    Row<T>::unpack(q[b], z);
#pragma unroll
    for (int e = 0; e < kVec; e += 2)
      e2[e / 2 & 1] = __fadd2_rn(e2[e / 2 & 1], row_exp2_pair(z[e], z[e + 1], r.m, c2));
  }
  e2[0] = __fadd2_rn(e2[0], e2[1]);
  if (kExact)
    r.s = summed(r.s, e2[0].x + e2[0].y, r.c);
  else
    r.s += e2[0].x + e2[0].y;
}

// A vector with its element e (-1: none) in place of what it had.
__device__ __forceinline__ uint4 with_element(const uint4& q, int e, float g) {
  const uint32_t x = __float_as_uint(g);
  return make_uint4(e == 0 ? x : q.x, e == 1 ? x : q.y, e == 2 ? x : q.z, e == 3 ? x : q.w);
}
__device__ __forceinline__ uint4 with_element(const uint4& q, int e, __nv_bfloat16 g) {
  const uint32_t x = __bfloat16_as_ushort(g), both = x | x << 16, keep = e & 1 ? 0x0000ffffu : 0xffff0000u;
  const auto word = [&](uint32_t w, int i) { return e >> 1 == i ? (w & keep) | (both & ~keep) : w; };
  return make_uint4(word(q.x, 0), word(q.y, 1), word(q.z, 2), word(q.w, 3));
}

// 16 bytes that start `shift` bytes (a multiple of the element's size, uniform) into
// the 32 of a and b.
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int shift) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (shift & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (shift & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const int bits = (shift & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                    __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// kLate: the form in which a test has a CTA come late, under a shorter limit.
constexpr uint64_t kLateLimitNs = 200000000ull;

template <typename T, bool kGrad, TokenEnds kEnds, bool kLate = false>
__global__ void __launch_bounds__(kGrad ? 128 : 256, kGrad ? 5 : 4)
    token_rows_kernel(const __grid_constant__ TokenParams p, const __grid_constant__ TokenPlan plan) {
  constexpr int kVec = Row<T>::kVec;
  constexpr bool kEdges = kEnds != kWhole;
  using S = Span<T, kEdges>;
  const float inf = __builtin_huge_valf();
  extern __shared__ __align__(16) unsigned char token_smem[];
  __shared__ TokenShared sh;
  const int ctas = plan.ctas, tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = nt >> 5;
  const int rank = ctas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int cluster = blockIdx.x / ctas, clusters = gridDim.x / ctas;
  const int batch = kBatch * nt;  // vectors
  const int chunk = row_chunk(p.V, ctas);
  const int lo = min(p.V, rank * chunk), hi = min(p.V, lo + chunk);
  const float c2 = __fdiv_rn(kRowLog2e, p.tau);
  const int own = warp * 32 * kBatch + lane;  // of a batch's vectors the thread's are own + 32 b
  uint4* const ring = reinterpret_cast<uint4*>(token_smem) + own;  // item b of place k at ring[k batch + 32 b]
  const int ring_end = plan.ring * batch;
  grid_dependency_wait();
  if (ctas > 1) {
    if (tid == 0) {
      mbar_init(&sh.full[0], 1);
      mbar_init(&sh.full[1], 1);
      sh.deaf = 0;
      fence_mbar_init();
    }
    __syncwarp();
    cluster_sync();  // peers' shared memory and barriers are there
  }

  const auto row_at = [&](long long r) { return static_cast<const T*>(p.logits) + r * p.ld; };
  const int batch_log = 31 - __clz(batch);  // (a power of two)
  const auto owns = [&](int v) { return (v & (batch - 1) & ~(32 * (kBatch - 1))) == own; };
  const auto item_of = [&](int v) { return v >> 5 & (kBatch - 1); };
  // Vectors at a slice's ends hold elements of its neighbours, which their thread makes -inf
  // when they are there; only what lies in front of or behind all logits is not read.
  const char* const front = static_cast<const char*>(p.logits);
  const char* const behind = front + ((p.M - 1) * p.ld + p.V) * static_cast<long long>(sizeof(T));
  const auto begins_before = [&](const S& s) { return kEdges && reinterpret_cast<const char*>(s.src) < front; };
  const auto ends_behind = [&](const S& s) {
    return kEdges && reinterpret_cast<const char*>(s.src + s.n_vec) > behind;
  };
  // A cluster's rows, one of each `clusters` in turn and not always the same one: rows
  // that take no part often follow a pattern, and every cluster should have its share.
  const auto row_in = [&](int turn) {
    return static_cast<long long>(turn) * clusters + (cluster + turn) % clusters;
  };
  const int turns = (p.M + clusters - 1) / clusters;
  // Tokens of 32 turns, one to a lane, and the turns that take part, a bit each; and of
  // the next 32, which come meanwhile.
  int token, token_next;
  float weight_next;
  unsigned live_now, live_next = 0;
  const auto fetch = [&](int turn, int& t, float& w) {
    const long long r = row_in(turn);
    const bool is = turn < turns && r < p.M;
    t = is ? p.token[r] : -1;
    w = is && p.weight ? p.weight[r] : 1.0f;
  };
  const auto taking_part = [&](int t, float w) {
    return __ballot_sync(0xffffffffu, t >= 0 && t < p.V && w != 0.0f);
  };
  fetch(lane, token, weight_next);
  live_now = taking_part(token, weight_next);
  fetch(32 + lane, token_next, weight_next);
  // The next batch to ask for, of the row in turn or of one of the two after it.
  int ask_batch = 0, ask_turn = 0, ask_place = 0, ask_first, ask_inner;
  unsigned ask_live = live_now & 1u;
  long long ask_row = row_in(0);
  const uint4* ask_src;
  int base = 0;  // the turn of lane 0's token
  const auto ask_begin = [&]() {
    const S s(row_at(ask_row), lo, hi);
    ask_first = begins_before(s) ? 1 : 0;
    ask_inner = s.n_vec - (ends_behind(s) ? 1 : 0) >> batch_log;
    ask_src = s.src + own;
  };
  if (ask_row < p.M) ask_begin();
  // A slice's last batch, with places that have no vector: -inf; or the first of all
  // logits.
  const auto ask_ends = [&]() {
    const T* row = row_at(ask_row);
    const S s(row, lo, hi);
    const int from = begins_before(s) ? 1 : 0, to = s.n_vec - (ends_behind(s) ? 1 : 0);
#pragma unroll 1
    for (int b = 0; b < kBatch; ++b) {
      const int v = own + ask_batch * batch + b * 32;
      uint4* slot = ring + ask_place + b * 32;
      if (v >= from && v < to) {
        copy_async16(slot, s.src + v);
      } else {
        uint4 q;
        T* d = reinterpret_cast<T*>(&q);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const int i = s.index(v) + e;
          d[e] = kEdges && v < s.n_vec && i >= lo && i < hi ? row[i] : Row<T>::neg_inf();
        }
        *slot = q;
      }
    }
  };
  const auto ask_one = [&]() {
    if (ask_live) {
      if (p.policy && ask_batch == 0 && tid < 4) {  // what the loss needs beside the logits
        const float* from = tid == 0 ? p.old_logp : tid == 1 ? p.advantage : tid == 2 ? p.ref_logp : p.weight;
        if (from) copy_async4(reinterpret_cast<float*>(&sh.row[ask_turn & 3]) + tid, from + ask_row);
      }
      if ((!kEdges || ask_batch >= ask_first) && ask_batch < ask_inner) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) copy_async16(ring + ask_place + b * 32, ask_src + b * 32);
      } else {
        ask_ends();
      }
    }
    copy_commit();
    ask_src += batch;
    ask_place += batch;
    if (ask_place == ring_end) ask_place = 0;
    if (++ask_batch == plan.batches) {
      ask_batch = 0;
      ++ask_turn;
      ask_row = row_in(ask_turn);
      ask_live = (ask_turn - base < 32 ? live_now >> (ask_turn - base) : live_next >> (ask_turn - base - 32)) & 1u;
      if (ask_live) ask_begin();
    }
  };
#pragma unroll 1
  for (int k = 0; k < plan.ring; ++k) ask_one();

  int place = 0;  // of the next batch to work on
  int heard_rows = 0;  // that take part
  bool deaf = false;   // (a warp's lanes alike)
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    if (turn - base == 32) {
      base = turn;
      token = token_next;
      live_now = live_next;
      fetch(turn + 32 + lane, token_next, weight_next);
    }
    if (turn - base == 16) live_next = taking_part(token_next, weight_next);  // (they are here by now)
    const long long r = row_in(turn);
    const bool live = live_now >> (turn - base) & 1u;
    const int t = __shfl_sync(0xffffffffu, token, turn - base);
    float up = 0.0f, m = 0.0f, s = 0.0f, loss = 0.0f, by = 0.0f, logp = 0.0f, zt = 0.0f, rest = 0.0f;
    const T* row = row_at(r);
    if (live) {
      const int buf = heard_rows & 1;
      // Where the token's logit lies, if in this CTA's slice: batch, thread, element.
      const S slice(row, lo, hi);
      const int place_t = t >= lo && t < hi ? t - slice.index(0) : -1;
      const int v_t = place_t / kVec;
      const bool mine = place_t >= 0 && owns(v_t);
      // The last vector's elements that are the slice's, 0: all; that vector, if this thread's.
      const int left = (slice.skip + hi - lo) % kVec, last_v = slice.n_vec - 1;
      const int cut = kEdges && left && owns(last_v) ? last_v : -1;
      RowSum sum{-inf, 0.0f, 0.0f};
      if (kGrad) copy_wait(plan.ring - plan.batches);
      int at = place;
#pragma unroll 1
      for (int j = 0; j < plan.batches; ++j) {
        if (!kGrad) copy_wait(plan.ring - 1);
        uint4* slot = ring + at;
        if (kEdges && j == 0 && tid < slice.first) {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (e < slice.skip) reinterpret_cast<T*>(slot)[e] = Row<T>::neg_inf();
        }
        if (kEdges && cut >> batch_log == j) {
          T* d = reinterpret_cast<T*>(slot + item_of(cut) * 32);
#pragma unroll
          for (int e = 1; e < kVec; ++e)
            if (e >= left) d[e] = Row<T>::neg_inf();
        }
        uint4 q[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) q[b] = slot[b * 32];
        if (mine && v_t >> batch_log == j)
          zt = Row<T>::to_float(reinterpret_cast<const T*>(slot + item_of(v_t) * 32)[place_t % kVec]);
        at += batch;
        if (at == ring_end) at = 0;
        add_batch<T, !kGrad>(sum, q, c2);
        if (!kGrad) ask_one();
      }
      if (!kGrad) place = at;
      __syncwarp();
      sum = warp_merged<!kGrad>(sum, c2);
      if (ctas > 1 && !deaf) {
        if (kLate && turn == plan.late_turn && cluster == 0 && rank == ctas - 1) pause_ns(3 * kLateLimitNs);
        if (lane < ctas) tell(&sh.part[buf][rank * warps + warp], &sh.full[buf], lane, sum);
        if (mine)
#pragma unroll 1
          for (int k = 0; k < ctas; ++k) tell(&sh.zt[buf], &sh.full[buf], k, zt);
        if (p.policy && tid < 4)
          tell(reinterpret_cast<float*>(&sh.info[buf]) + tid, &sh.full[buf], rank,
               reinterpret_cast<const float*>(&sh.row[turn & 3])[tid]);
        if (tid == 0) mbar_arrive_expect_tx(&sh.full[buf], ctas * warps * 16 + 4 + (p.policy ? 16 : 0));
        __syncwarp();
        const bool here = heard(&sh.full[buf], heard_rows >> 1 & 1, &sh.deaf, kLate ? kLateLimitNs : kWaitLimitNs);
        deaf = __any_sync(0xffffffffu, !here || any_deaf(&sh.deaf));
        if (deaf && lane < ctas) tell_deaf(&sh.deaf, lane);
      } else if (ctas == 1) {
        if (mine) sh.zt[buf] = zt;
        if (p.policy && tid < 4)
          reinterpret_cast<float*>(&sh.info[buf])[tid] = reinterpret_cast<const float*>(&sh.row[turn & 3])[tid];
        if (lane == 0) sh.part[buf][warp] = make_float4(sum.m, sum.s, sum.c, 0.0f);
        __syncthreads();
      }
      ++heard_rows;
      sum = RowSum{-inf, 0.0f, 0.0f};
#pragma unroll 1
      for (int k = lane; k < ctas * warps; k += 32) {
        const float4 x = sh.part[buf][k];
        sum = merged(sum, RowSum{x.x, x.y, x.z}, c2);
      }
      __syncwarp();
      sum = warp_merged<!kGrad>(sum, c2);
      m = deaf ? __int_as_float(0x7fc00000) : sum.m;
      s = deaf ? __int_as_float(0x7fc00000) : sum.s + sum.c;
      rest = (sum.s - s) + sum.c;
      zt = sh.zt[buf];
      logp = token_logp_of(zt, m, s, p.tau);
      if (p.policy && (kGrad || tid == 0)) {
        policy_terms(p, sh.info[buf], logp, loss, by);
        up = __fdiv_rn(by, p.tau);
      }
      __syncwarp();
    } else if (!kGrad) {
#pragma unroll 1
      for (int j = 0; j < plan.batches; ++j) {
        ask_one();
        place += batch;
        if (place == ring_end) place = 0;
      }
    }
    if (rank == 0 && tid == 0 && r < p.M) {
      p.logp[r] = live ? token_logp_written(zt, m, s, rest, p.inv_tau) : 0.0f;
      p.stats[2 * r] = m;
      p.stats[2 * r + 1] = s;
      if (p.policy) {
        p.loss[r] = loss;
        p.slope[r] = by;
      }
    }
    if (kGrad && r < p.M) {
      const S span(row, lo, hi);
      T* grow = static_cast<T*>(p.grad) + r * p.ld_grad;
      // The 16 bytes of the gradient's that vector 0 begins in, `apart` elements before it.
      const uintptr_t at0 = reinterpret_cast<uintptr_t>(grow + span.index(0));
      const int apart = kEnds == kShifted ? static_cast<int>((at0 & 15) / sizeof(T)) : 0;
      uint4* dst = reinterpret_cast<uint4*>(at0 & ~static_cast<uintptr_t>(15)) + own;
      const int whole = span.last >> batch_log;  // batches of vectors that are the row's, the first perhaps not
      const float k = up == 0.0f ? 0.0f : __fdiv_rn(-up, s);
#pragma unroll 1
      for (int j = 0; j < plan.batches; ++j) {
        const uint4* slot = ring + place;
        uint4 q[kBatch];
        if (up == 0.0f) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) q[b] = make_uint4(0u, 0u, 0u, 0u);
        } else {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            float z[kVec];
            Row<T>::unpack(slot[b * 32], z);
#pragma unroll
            for (int e = 0; e < kVec; e += 2) {
              const float2 g = __fmul2_rn(make_float2(k, k), row_exp2_pair(z[e], z[e + 1], m, c2));
              z[e] = g.x;
              z[e + 1] = g.y;
            }
            q[b] = Row<T>::pack(z);
          }
        }
        place += batch;
        if (place == ring_end) place = 0;
        if constexpr (kEnds == kShifted) {
          const int v_t = (t - span.index(0)) / kVec;
          if (up != 0.0f && t >= lo && t < hi && v_t >> batch_log == j && owns(v_t)) {
            const float g = fmaf(k, token_share(zt, m, c2), up);
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
              q[b] = with_element(q[b], b == item_of(v_t) ? (t - span.index(0)) % kVec : -1, Row<T>::from_float(g));
          }
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            // The vector before; the warp's first has none.
            const uint4 give = lane == 31 && b > 0 ? q[b > 0 ? b - 1 : 0] : q[b];
            const int from = (lane + 31) & 31;
            const uint4 prev = make_uint4(__shfl_sync(0xffffffffu, give.x, from), __shfl_sync(0xffffffffu, give.y, from),
                                          __shfl_sync(0xffffffffu, give.z, from), __shfl_sync(0xffffffffu, give.w, from));
            const uint4 out = apart ? shifted(prev, q[b], 16 - apart * static_cast<int>(sizeof(T))) : q[b];
            const int i0 = span.index(own + j * batch + b * 32) - apart;  // the first element of those 16 bytes
            const bool known = b > 0 || lane > 0 || apart == 0;
            if (known && i0 >= lo && i0 + kVec <= hi) {
              __stcs(dst + b * 32, out);
            } else if (!known && i0 + apart >= lo && i0 + kVec <= hi) {
              store_from(reinterpret_cast<T*>(dst + b * 32), out, apart);
            } else {
              const T* d = reinterpret_cast<const T*>(&out);
#pragma unroll
              for (int e = 0; e < kVec; ++e)
                if (i0 + e >= lo && i0 + e < hi && (known || e >= apart)) grow[i0 + e] = d[e];
            }
            if (b == kBatch - 1 && lane == 31) {  // and the warp's last, in the 16 bytes of the vector behind
              const uint4 last = shifted(q[b], q[b], 16 - apart * static_cast<int>(sizeof(T)));
              const int i = i0 + kVec;  // of that
              if (i >= lo && i + apart <= hi) {
                if (apart) store_front(reinterpret_cast<T*>(dst + b * 32 + 1), last, apart);
              } else {
                const T* d = reinterpret_cast<const T*>(&last);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                  if (e < apart && i + e >= lo && i + e < hi) grow[i + e] = d[e];
              }
            }
          }
        } else if (j < whole) {
          if (kEdges && j == 0 && tid < span.first) {
            const T* d = reinterpret_cast<const T*>(&q[0]);
#pragma unroll
            for (int e = 1; e < kVec; ++e)
              if (e >= span.skip) grow[lo - span.skip + e] = d[e];
          } else {
            __stcs(dst, q[0]);
          }
#pragma unroll
          for (int b = 1; b < kBatch; ++b) __stcs(dst + b * 32, q[b]);
        } else {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const int v = own + j * batch + b * 32;
            if (v >= span.first && v < span.last) {
              __stcs(dst + b * 32, q[b]);
            } else if (kEdges && v < span.n_vec) {
              const T* d = reinterpret_cast<const T*>(&q[b]);
#pragma unroll
              for (int e = 0; e < kVec; ++e) {
                const int i = span.index(v) + e;
                if (i >= lo && i < hi) grow[i] = d[e];
              }
            }
          }
        }
        dst += batch;
        ask_one();
      }
      // The token's own element, by the thread that has just written its vector.
      if (kEnds != kShifted && up != 0.0f && t >= lo && t < hi && owns((t - span.index(0)) / kVec))
        grow[t] = Row<T>::from_float(fmaf(k, token_share(zt, m, c2), up));
    }
  }
  grid_launch_dependents();
  if (ctas > 1) {
    // Nothing is on its way into a CTA that leaves: every row's sums were heard of, or what was
    // told to the deaf, before it was known that they are, has had its time.
    if (deaf || any_deaf(&sh.deaf)) pause_ns(1000000);
    __syncwarp();
    cluster_sync();
  }
}

// Gradient rows from the stats: elements [lo, hi) of row r, every one written.
template <typename T, int kFlight>
__device__ __forceinline__ void token_grad_part(const T* row, T* grow, int lo, int hi, int t, float up, float m,
                                                float s, float c2, int tid, int nt) {
  constexpr int kVec = Row<T>::kVec;
  const Span<T> out(grow, lo, hi);
  uint4* dst = const_cast<uint4*>(out.src);
  const auto stored = [&](int v, const uint4& q) { __stcs(dst + v, q); };
  if (up == 0.0f) {
#pragma unroll 1
    for (int v = out.first + tid; v < out.last; v += nt) stored(v, make_uint4(0u, 0u, 0u, 0u));
    if (tid < out.ends()) grow[out.end(tid)] = Row<T>::from_float(0.0f);
    return;
  }
  const float k = __fdiv_rn(-up, s);  // times e_v
  const auto element = [&](float z, int i) { return fmaf(k, token_share(z, m, c2), i == t ? up : 0.0f); };
  const auto vector = [&](int v, const uint4& q) {
    float z[kVec];
    Row<T>::unpack(q, z);
#pragma unroll
    for (int e = 0; e < kVec; e += 2) {
      const float2 g = __fmul2_rn(make_float2(k, k), row_exp2_pair(z[e], z[e + 1], m, c2));
      z[e] = g.x;
      z[e + 1] = g.y;
    }
    const unsigned at = static_cast<unsigned>(t - out.index(v));
    if (at < static_cast<unsigned>(kVec)) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) z[e] += at == e ? up : 0.0f;
    }
    stored(v, Row<T>::pack(z));
  };
  const uintptr_t in = reinterpret_cast<uintptr_t>(row + out.index(0));
  const int shift = static_cast<int>(in & 15);
  const uint4* src = reinterpret_cast<const uint4*>(in & ~static_cast<uintptr_t>(15));
  // Where logits and gradient lie differently, a vector takes parts of two, and
  // those of the row's ends may reach outside it.
  int first = out.first, last = out.last;
  if (shift) {
    if (out.index(first) - lo < shift / static_cast<int>(sizeof(T))) ++first;
    if (hi - out.index(last) < kVec - shift / static_cast<int>(sizeof(T))) --last;
    if (last < first) last = first;
  }
  if (!shift) {
    for_vectors<kFlight, false>(src, first + tid, last, nt, vector);
  } else {
#pragma unroll 1
    for (int v = first + tid; v < last; v += kFlight * nt) {
      uint4 a[kFlight], b[kFlight];
#pragma unroll
      for (int j = 0; j < kFlight; ++j)
        if (v + j * nt < last) {
          a[j] = __ldg(src + v + j * nt);
          b[j] = __ldg(src + v + j * nt + 1);
        }
#pragma unroll
      for (int j = 0; j < kFlight; ++j)
        if (v + j * nt < last) vector(v + j * nt, shifted(a[j], b[j], shift));
    }
  }
  // The elements beside the vectors, at most three vectors' at either end.
  const int head = last > first ? out.index(first) - lo : hi - lo;
  const int tail = last > first ? out.index(last) : hi;
#pragma unroll 1
  for (int i = tid; i < head + hi - tail; i += nt) {
    const int e = i < head ? lo + i : tail + i - head;
    grow[e] = Row<T>::from_float(element(Row<T>::to_float(row[e]), e));
  }
}

// Gradients alone: `parts` CTAs to a row, `chunk` elements each; nothing waits for
// anything, HBM bounds it: 2048 rows of 126464 bf16 155 us, of 152 at the copy's rate.
template <typename T>
__global__ void __launch_bounds__(256)
    token_grad_kernel(const __grid_constant__ TokenParams p, int parts, int chunk) {
  const int r = blockIdx.x / parts, part = blockIdx.x % parts;
  grid_dependency_wait();
  const int t = p.token[r];
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  T* grow = static_cast<T*>(p.grad) + static_cast<long long>(r) * p.ld_grad;
  const float c2 = __fdiv_rn(kRowLog2e, p.tau);
  const float m = p.stats[2ll * r], s = p.stats[2ll * r + 1];
  const float slope = p.slope ? p.slope[r] : 1.0f, above = p.upstream ? p.upstream[r] : 1.0f;
  const bool live = t >= 0 && t < p.V && slope != 0.0f && above != 0.0f;
  const float up = live ? __fdiv_rn(slope * above, p.tau) : 0.0f;
  const int lo = part * chunk, hi = min(p.V, lo + chunk);
  if (lo < hi) token_grad_part<T, 4>(row, grow, lo, hi, t, up, m, s, c2, threadIdx.x, blockDim.x);
}

// ---------------------------------------------------------- pairs of sequences --

struct PairParams {
  const float *logp, *ref_logp, *weight;
  const int32_t* offsets;  // [2 pairs + 1]
  int M, pairs;
  float beta, smoothing;
  const float* upstream;  // [pairs] or null
  float *loss, *margin;
  float* grad_logp;       // [M] or null
};

constexpr int kPairThreads = 256;

// A CTA to a pair; one more for the rows in no sequence.  Latency: two dependent
// loads, a reduction and the writes, 6 us for 8 pairs of 250 rows.
__global__ void __launch_bounds__(kPairThreads) preference_kernel(const __grid_constant__ PairParams p) {
  __shared__ double part[kPairThreads / 32];
  const int tid = threadIdx.x, i = blockIdx.x;
  grid_dependency_wait();
  grid_launch_dependents();
  const auto at = [&](long long k) { return min(max(p.offsets[k], 0), p.M); };
  if (i == p.pairs) {
    if (!p.grad_logp) return;
    const int lo = at(0), hi = at(2ll * p.pairs);
#pragma unroll 1
    for (int r = tid; r < p.M; r += kPairThreads)
      if (r < lo || r >= hi) p.grad_logp[r] = 0.0f;
    return;
  }
  const int a = at(2ll * i), b = max(a, at(2ll * i + 1)), c = max(b, at(2ll * i + 2));
  double sum = 0.0;
#pragma unroll 1
  for (int r = a + tid; r < c; r += kPairThreads) {
    const float w = p.weight ? p.weight[r] : 1.0f;
    if (w == 0.0f) continue;
    const double x = static_cast<double>(w) * (static_cast<double>(p.logp[r]) - (p.ref_logp ? p.ref_logp[r] : 0.0f));
    sum += r < b ? x : -x;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) part[tid >> 5] = sum;
  __syncthreads();
  sum = part[0];
#pragma unroll
  for (int k = 1; k < kPairThreads / 32; ++k) sum += part[k];
  const float margin = static_cast<float>(static_cast<double>(p.beta) * sum);
  const float e = expf(-fabsf(margin));              // in (0, 1]
  const float down = (margin >= 0.0f ? e : 1.0f) / (1.0f + e);  // sigmoid(-margin)
  if (tid == 0) {
    // -log sigmoid(x) = log(1 + exp(-|x|)) + max(-x, 0): of the two terms one has the |x|.  (A
    // margin is infinite where a token is suppressed; a share of 0 has no term.)
    const float share = margin < 0.0f ? 1.0f - p.smoothing : p.smoothing;
    p.loss[i] = margin != margin ? margin : log1pf(e) + (share != 0.0f ? share * fabsf(margin) : 0.0f);
    p.margin[i] = margin;
  }
  if (!p.grad_logp) return;
  const float up = (p.upstream ? p.upstream[i] : 1.0f) * p.beta * (p.smoothing - down);
#pragma unroll 1
  for (int r = a + tid; r < c; r += kPairThreads) {
    const float w = p.weight ? p.weight[r] : 1.0f;
    p.grad_logp[r] = w == 0.0f ? 0.0f : (r < b ? up : -up) * w;
  }
}

}  // namespace cai
