// Distillation from a teacher's top logits (cai_distill_loss,
// cai_distill_backward).
//
// p = softmax(z / tau) over the vocabulary, q the teacher's probabilities of the
// tokens in its record.  Without the teacher's log-sum-exp q is renormalised
// over the record; with it the rest q_r = 1 - sum q is one more class, which the
// student's p_r = sum of p outside the record answers.
//   loss = w tau^2 [ sum_k q_k (log q_k - log p_k) + q_r (log q_r - log p_r) ]
//   dloss/dz_v = w tau (A p_v - q_v)            in the record
//              = w tau (A p_r - q_r) p_v / p_r  outside,   A = sum q + q_r.
// p_r is summed over the tokens outside, never 1 minus the others: once the
// slice is in shared memory the record's logits are taken out of it and -inf
// left in their places, so the pass over the slice sees the rest alone.
#pragma once

#include "row_ops.cuh"
#include "sample.cuh"
#include "softmax.cuh"

namespace cai {

struct DistillParams {
  const void* logits;
  long long ld;
  int M, V, K;
  float tau;
  const float* top_values;    // [M, K]
  const int32_t* top_index;   // [M, K], outside [0, V): no entry
  const float* top_lse;       // [M] or null
  const float* weight;        // [M] or null
  float* loss;                // [M], null in the backward call
  float* stats;               // [M, 2]: written by the loss, read by the backward call
  const float* upstream;      // [M], the backward call's dL/dloss; null otherwise
  void* grad;                 // [M, ld_grad] or null
  long long ld_grad;
};

constexpr float kLn2 = 0.6931471805599453f;

// Running maximum and sum of 2^(x - max).
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  // -inf on both sides: no element yet.
  const float ea = a.m == m ? 1.0f : fast_exp2(a.m - m);
  const float eb = b.m == m ? 1.0f : fast_exp2(b.m - m);
  return MaxSum{m, a.s * ea + b.s * eb};
}
__device__ __forceinline__ unsigned long long bits_of(MaxSum a) {
  return (static_cast<unsigned long long>(__float_as_uint(a.s)) << 32) | __float_as_uint(a.m);
}
__device__ __forceinline__ MaxSum max_sum_of(unsigned long long b) {
  return MaxSum{__uint_as_float(static_cast<uint32_t>(b)),
                __uint_as_float(static_cast<uint32_t>(b >> 32))};
}
struct MaxSumOp {
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return bits_of(merge(max_sum_of(a), max_sum_of(b)));
  }
};

// What a CTA keeps of the teacher's record.
struct Record {
  float q[kTopMax];      // probability (of its token, in the entry that speaks for it)
  float logq[kTopMax];
  float z[kTopMax];      // the student's logit, of the entries in this CTA's slice
  float token_q[kTopMax];
  int at[kTopMax];       // element of the row, -1: no entry
  float scratch[kRowMaxWarps];
  float loss_part[kRowMaxCluster];
};

template <typename Op>
__device__ __forceinline__ float cta_float(float* scratch, float v, Op op) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = scratch[0];
  for (int i = 1; i < static_cast<int>(blockDim.x >> 5); ++i) r = op(r, scratch[i]);
  return r;
}

// Marks in place of an element: an index below 2^16 as bits of the element's
// type (never read as a value).
__device__ __forceinline__ float mark_of(int k, float) { return __uint_as_float(k); }
__device__ __forceinline__ __nv_bfloat16 mark_of(int k, __nv_bfloat16) {
  return __ushort_as_bfloat16(static_cast<unsigned short>(k));
}
__device__ __forceinline__ int of_mark(float x) { return static_cast<int>(__float_as_uint(x)); }
__device__ __forceinline__ int of_mark(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }

template <typename T>
__global__ void __launch_bounds__(kRowMaxThreads)
    distill_kernel(const __grid_constant__ DistillParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  __shared__ RowShared sh;
  __shared__ Record rec;
  row_begin();
  RowCta c{&sh, static_cast<int>(cluster_ctarank()), ctas, 0};
  const int r = blockIdx.x / ctas, tid = threadIdx.x, nt = blockDim.x;
  const float inf = __uint_as_float(0x7f800000u);
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  T* grow = static_cast<T*>(p.grad) + static_cast<long long>(r) * p.ld_grad;
  const Slice<T> s = row_slice(row, p.V, c.rank, ctas, slice_smem);
  const bool backward = p.upstream != nullptr;
  const float w = p.weight ? p.weight[r] : 1.0f;

  // The record: probabilities of its entries, the same in every CTA.
  float high = -inf;
  for (int k = tid; k < p.K; k += nt) {
    const int at = p.top_index[static_cast<long long>(r) * p.K + k];
    const float t = __fdiv_rn(p.top_values[static_cast<long long>(r) * p.K + k], p.tau);
    const bool given = at >= 0 && at < p.V;
    rec.at[k] = given ? at : -1;
    rec.logq[k] = given ? t : -inf;
    if (given) high = fmaxf(high, t);
  }
  const auto max_op = [](float a, float b) { return fmaxf(a, b); };
  const auto add_op = [](float a, float b) { return a + b; };
  bool any = false;
  for (int k = tid; k < p.K; k += nt) any |= rec.at[k] >= 0;
  const bool live = w != 0.0f && __syncthreads_or(any);
  if (!live) {  // the same in the whole cluster; the row is not read
    if (p.grad)
      for (int i = s.lo + tid; i < s.hi; i += nt) grow[i] = Row<T>::from_float(0.0f);
    if (c.rank == 0 && tid == 0 && p.loss) {
      p.loss[r] = 0.0f;
      p.stats[2ll * r] = 0.0f;
      p.stats[2ll * r + 1] = 0.0f;
    }
    row_begun();
    return;
  }
  load_slice<T, 4>(s, row, [](const uint4&) {});
  row_begun();
  // log q = (t - from) - norm, the larger of the two subtracted first.
  float from = 0.0f, norm;
  if (p.top_lse) {
    norm = p.top_lse[r];
  } else {
    from = cta_float(rec.scratch, high, max_op);
    float sum = 0.0f;
    for (int k = tid; k < p.K; k += nt) sum += expf(rec.logq[k] - from);
    norm = logf(cta_float(rec.scratch, sum, add_op));
  }
  float qsum = 0.0f;
  for (int k = tid; k < p.K; k += nt) {
    const float lq = (rec.logq[k] - from) - norm;
    const float q = rec.at[k] >= 0 ? expf(lq) : 0.0f;
    rec.logq[k] = lq;
    rec.q[k] = q;
    qsum += q;
  }
  qsum = cta_float(rec.scratch, qsum, add_op);  // also: the slice is in place
  const float rest = p.top_lse ? fmaxf(1.0f - qsum, 0.0f) : 0.0f;
  const float whole = qsum + rest;

  // Take the record's logits out of the slice.  An entry that finds its own mark
  // in its place speaks for its token.
  for (int k = tid; k < p.K; k += nt) {
    const int at = rec.at[k];
    if (at >= s.lo && at < s.hi) rec.z[k] = Row<T>::to_float(s.data[at - s.lo]);
  }
  __syncthreads();
  for (int k = tid; k < p.K; k += nt) {
    const int at = rec.at[k];
    if (at >= s.lo && at < s.hi) s.data[at - s.lo] = mark_of(k, T());
  }
  __syncthreads();
  static_assert(kTopMax / 128 <= 32, "one bit for each entry of a thread");
  uint32_t speaks = 0;  // bit j: entry tid + j nt speaks for its token
  bool twice = false;
  for (int k = tid, j = 0; k < p.K; k += nt, ++j) {
    const int at = rec.at[k];
    if (at >= s.lo && at < s.hi) {
      if (of_mark(s.data[at - s.lo]) == k)
        speaks |= 1u << j;
      else
        twice = true;
    }
  }
  if (__syncthreads_or(twice)) {
    // Some token is named more than once: its first entry speaks, with the
    // entries' probabilities added up in their order.
    speaks = 0;
    for (int k = tid, j = 0; k < p.K; k += nt, ++j) {
      const int at = rec.at[k];
      if (at < s.lo || at >= s.hi) continue;
      bool first = true;
      float q = 0.0f;
      for (int i = 0; i < p.K; ++i)
        if (rec.at[i] == at) {
          first &= i >= k;
          q += rec.q[i];
        }
      if (first) speaks |= 1u << j;
      rec.token_q[k] = q;
    }
    __syncthreads();
    for (int k = tid, j = 0; k < p.K; k += nt, ++j)
      if (speaks >> j & 1u) rec.q[k] = rec.token_q[k];
  }
  for (int k = tid, j = 0; k < p.K; k += nt, ++j)
    if (speaks >> j & 1u) s.data[rec.at[k] - s.lo] = Row<T>::neg_inf();
  __syncthreads();

  // The sums of 2^x, x = z log2(e) / tau, over the record and over the rest, each
  // relative to a reference of its own: its maximum, and in the backward call
  // the logarithm that the forward call left.  The backward call adds them up
  // again, since a logarithm of about 20 in fp32 holds p to 1e-6 only.
  const float c2 = __fdiv_rn(kRowLog2e, p.tau);
  MaxSum in{-inf, 0.0f}, out{-inf, 0.0f};
  if (backward) {
    in.m = p.stats[2ll * r] * kRowLog2e;
    out.m = p.stats[2ll * r + 1] * kRowLog2e;
  }
  for (int k = tid, j = 0; k < p.K; k += nt, ++j)
    if (speaks >> j & 1u) {
      if (backward) {
        in.s += fast_exp2(fmaf(rec.z[k], c2, -in.m));
      } else {
        const float x = rec.z[k] * c2;
        in = merge(in, MaxSum{x, x == -inf ? 0.0f : fast_exp2(fmaf(rec.z[k], c2, -x))});
      }
    }
  for (int v = tid; v < s.n_vec; v += nt) {
    float z[kVec];
    Row<T>::unpack(s.vec[v], z);
    if (!backward) {
      float m = z[0];
#pragma unroll
      for (int e = 1; e < kVec; ++e) m = max_nan(m, z[e]);
      m *= c2;
      if (!(m <= out.m)) {  // a new maximum, or NaN
        out.s = out.m == -inf ? 0.0f : out.s * fast_exp2(out.m - m);
        out.m = m;
      }
    }
    if (out.m != -inf) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) out.s += fast_exp2(fmaf(z[e], c2, -out.m));
    }
  }
  out = max_sum_of(cluster_reduce(c, bits_of(out), MaxSumOp()));
  in = max_sum_of(cluster_reduce(c, bits_of(in), MaxSumOp()));
  const MaxSum all = merge(out, in);
  const float ref = out.m == -inf ? 0.0f : out.m;
  const float log2_all = log2f(all.s);
  if (!backward) {
    float part = 0.0f;
    for (int k = tid; k < p.K; k += nt) {
      const int at = rec.at[k];
      if (at >= s.lo && at < s.hi) {
        const float q = expf(rec.logq[k]);
        if (q > 0.0f)
          part += q * (rec.logq[k] - (fmaf(rec.z[k], c2, -all.m) - log2_all) * kLn2);
      }
    }
    part = cta_float(rec.scratch, part, add_op);
    if (tid == 0) st_peer(reinterpret_cast<const uint32_t*>(&rec.loss_part[c.rank]), 0,
                          __float_as_uint(part));
    row_sync();
    if (c.rank == 0 && tid == 0) {
      float kl = 0.0f;
      for (int q = 0; q < ctas; ++q) kl += rec.loss_part[q];
      const float log_rest = ((out.m - all.m) + (log2f(out.s) - log2_all)) * kLn2;
      if (rest > 0.0f) kl += rest * (logf(rest) - log_rest);
      p.loss[r] = w * (p.tau * p.tau) * kl;
      p.stats[2ll * r] = (all.m + log2_all) * kLn2;
      p.stats[2ll * r + 1] = (out.m + log2f(out.s)) * kLn2;
    }
  }
  if (!p.grad) return;

  const float up = (backward ? w * p.upstream[r] : w) * p.tau;
  // The student's probability of the rest as one class; of its gradient each
  // token has its part.  Where the class has no probability nothing is divided.
  const float p_rest = out.m == -inf ? 0.0f : out.s * fast_exp2(out.m - all.m) / all.s;
  const float coef = out.s > 0.0f || out.s != out.s ? up * (whole * p_rest - rest) / out.s : 0.0f;
  const auto grad_of = [&](float z) { return coef * fast_exp2(fmaf(z, c2, -ref)); };
  const uint32_t a_in = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + s.lo)) & 15u;
  const uint32_t a_out = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(grow + s.lo)) & 15u;
  if (a_in == a_out) {
    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(grow + s.lo) &
                                          ~static_cast<uintptr_t>(15));
    for (int v = tid; v < s.n_vec; v += nt) {
      float z[kVec];
      Row<T>::unpack(s.vec[v], z);
#pragma unroll
      for (int e = 0; e < kVec; ++e) z[e] = grad_of(z[e]);
      const int i0 = s.index(v, 0);
      if (i0 >= s.lo && i0 + kVec <= s.hi) {
        dst[v] = Row<T>::pack(z);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (i0 + e >= s.lo && i0 + e < s.hi) grow[i0 + e] = Row<T>::from_float(z[e]);
      }
    }
  } else {
    for (int i = s.lo + tid; i < s.hi; i += nt)
      grow[i] = Row<T>::from_float(grad_of(Row<T>::to_float(s.data[i - s.lo])));
  }
  __syncthreads();  // the record's tokens, written as -inf above, come after
  for (int k = tid, j = 0; k < p.K; k += nt, ++j)
    if (speaks >> j & 1u) {
      const float pk = fast_exp2(fmaf(rec.z[k], c2, -all.m)) / all.s;
      grow[rec.at[k]] = Row<T>::from_float(up * (whole * pk - rec.q[k]));
    }
}

}  // namespace cai
