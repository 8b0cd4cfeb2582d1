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
// p_r is summed over the tokens outside, never 1 minus the others: a bitmap of the
// slice tells the pass over it which elements the record names.
#pragma once

#include <cstddef>

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

// Running maximum of logits and sum of 2^((z - max) c2).  The maximum is a logit, and
// differences are taken before the product: relative to a rounded max c2, the
// exponent of the maximum itself would be that product's rounding error, hundreds
// where |max c2| passes 2^31 and 10^30 at a type's lowest value.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ float share_of(float z, float from, float c2) {
  return fast_exp2(__fmul_rn(__fsub_rn(z, from), c2));
}
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c2) {
  const float m = fmaxf(a.m, b.m);
  // -inf on both sides: no element yet.
  const float ea = a.m == m ? 1.0f : share_of(a.m, m, c2);
  const float eb = b.m == m ? 1.0f : share_of(b.m, m, c2);
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
  float c2;
  __device__ __forceinline__ unsigned long long operator()(unsigned long long a,
                                                           unsigned long long b) const {
    return bits_of(merge(max_sum_of(a), max_sum_of(b), c2));
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
  const int n = blockDim.x >> 5;  // a power of two
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = scratch[threadIdx.x & (n - 1)];
#pragma unroll 1
  for (int o = n >> 1; o >= 1; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Bits of the slice's vectors, kVec for each: which elements the record names.
template <typename T>
__device__ __forceinline__ uint32_t vector_bits(const uint32_t* bits, int v) {
  constexpr int kVec = Row<T>::kVec;
  return (bits[v / (32 / kVec)] >> (v % (32 / kVec) * kVec)) & ((1u << kVec) - 1u);
}
__host__ __device__ __forceinline__ size_t bitmap_bytes(int slice_elems) {
  return (static_cast<size_t>(slice_elems) + 16 + 31) / 32 * 4;
}

// Dynamic shared memory: the slice (kCluster) or what is kept of the row, then the
// bitmap.  Loss and gradient in one call read a row once from HBM and write it once:
// 2048 rows of 126464 bf16, K = 64, of which one in eight has no weight and is not
// read, 216 us, 4.5 TB/s of 0.97 GB, 66 % of the copy's rate; the first pass and the
// second overlap between two CTAs on an SM only (the SMs issue on 62 % of the cycles,
// 139 instructions for 16 bytes, 87 of them for the loss).  All rows read: 235 us, the
// loss alone 150 and the backward call 229, of 152, 76 and 152 at the copy's rate.  33
// rows of 4099 float32, loss and gradient in two calls: 17 us, the host's.
template <typename T, bool kCluster>
__global__ void __launch_bounds__(512, kCluster ? 1 : 2)
    distill_kernel(const __grid_constant__ DistillParams p, int ctas) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ __align__(16) unsigned char slice_smem[];
  // (without its lists, which come last)
  __shared__ __align__(16) unsigned char shared_raw[offsetof(RowShared, listed)];
  RowShared& sh = *reinterpret_cast<RowShared*>(shared_raw);
  __shared__ Record rec;
  using Cta = RowCta<kCluster>;
  Cta::begin();
  Cta c(&sh, ctas);
  const int r = kCluster ? blockIdx.x / ctas : blockIdx.x, tid = threadIdx.x, nt = blockDim.x;
  const float inf = __uint_as_float(0x7f800000u);
  const T* row = static_cast<const T*>(p.logits) + static_cast<long long>(r) * p.ld;
  T* grow = static_cast<T*>(p.grad) + static_cast<long long>(r) * p.ld_grad;
  const Slice<T, kCluster> s =
      row_slice<T, kCluster>(row, p.V, c.rank(), c.ctas(), slice_smem, kCluster ? 0 : ctas, sh.edge);
  uint32_t* bits = reinterpret_cast<uint32_t*>(
      slice_smem + (kCluster ? row_slice_bytes(p.V, c.ctas(), sizeof(T)) : static_cast<size_t>(ctas) * 16));
  const bool backward = p.upstream != nullptr;
  const float w = p.weight ? p.weight[r] : 1.0f;
  const uint32_t a_in = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + s.lo)) & 15u;
  const uint32_t a_out = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(grow + s.lo)) & 15u;
  uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(grow + s.lo) &
                                        ~static_cast<uintptr_t>(15));

  // The record: probabilities of its entries, the same in every CTA; the
  // student's logits of those in this CTA's slice.
  float high = -inf;
  bool any = false;
  if (w != 0.0f)
#pragma unroll 1
    for (int k = tid; k < p.K; k += nt) {
      const int at = p.top_index[static_cast<long long>(r) * p.K + k];
      const float t = __fdiv_rn(p.top_values[static_cast<long long>(r) * p.K + k], p.tau);
      const bool given = at >= 0 && at < p.V;
      any |= given;
      rec.at[k] = given ? at : -1;
      rec.logq[k] = given ? t : -inf;
      rec.z[k] = given && s.holds(at) ? Row<T>::to_float(row[at]) : 0.0f;
      if (given) high = fmaxf(high, t);
    }
  const int n_bits = (s.n_vec * kVec + 31) / 32;
#pragma unroll 1
  for (int i = tid; i < n_bits; i += nt) bits[i] = 0;
  if (!__syncthreads_or(any)) {  // the same in the whole cluster; the row is not read
    if (p.grad) {
      if (a_in == a_out) {
#pragma unroll 1
        for (int v = tid; v < s.n_vec; v += nt)
          if (v >= s.first && v < s.last)
            dst[v] = make_uint4(0u, 0u, 0u, 0u);
          else
#pragma unroll 1
            for (int e = 0; e < kVec; ++e)
              if (s.holds(s.index(v) + e)) grow[s.index(v) + e] = Row<T>::from_float(0.0f);
      } else {
#pragma unroll 1
        for (int i = s.lo + tid; i < s.hi; i += nt) grow[i] = Row<T>::from_float(0.0f);
      }
    }
    if (c.rank() == 0 && tid == 0 && p.loss) {
      p.loss[r] = 0.0f;
      p.stats[2ll * r] = 0.0f;
      p.stats[2ll * r + 1] = 0.0f;
    }
    c.begun();
    return;
  }

  // Mark the record's tokens.  The entry that finds its token unmarked speaks for
  // it.
  static_assert(kTopMax / 64 <= 32, "one bit for each entry of a thread");
  uint32_t speaks = 0;  // bit j: entry tid + j nt speaks for its token
  bool twice = false;
#pragma unroll 1
  for (int k = tid, j = 0; k < p.K; k += nt, ++j) {
    const int at = rec.at[k];
    if (at >= 0 && s.holds(at)) {
      const uint32_t i = static_cast<uint32_t>(at - s.index(0)), bit = 1u << (i & 31u);
      if (atomicOr(&bits[i >> 5], bit) & bit)
        twice = true;
      else
        speaks |= 1u << j;
    }
  }
  const auto max_op = [](float a, float b) { return fmaxf(a, b); };
  const auto add_op = [](float a, float b) { return a + b; };
  // log q = (t - from) - norm, the larger of the two subtracted first.
  float from = 0.0f, norm;
  if (p.top_lse) {
    norm = p.top_lse[r];
  } else {
    from = cta_float(rec.scratch, high, max_op);
    float sum = 0.0f;
#pragma unroll 1
    for (int k = tid; k < p.K; k += nt) sum += expf(rec.logq[k] - from);
    norm = logf(cta_float(rec.scratch, sum, add_op));
  }
  float qsum = 0.0f;
#pragma unroll 1
  for (int k = tid; k < p.K; k += nt) {
    const float lq = (rec.logq[k] - from) - norm;
    const float q = rec.at[k] >= 0 ? expf(lq) : 0.0f;
    rec.logq[k] = lq;
    rec.q[k] = q;
    qsum += q;
  }
  qsum = cta_float(rec.scratch, qsum, add_op);  // also: the bits are set
  const float rest = p.top_lse ? fmaxf(1.0f - qsum, 0.0f) : 0.0f;
  const float whole = qsum + rest;
  if (__syncthreads_or(twice)) {
    // Some token is named more than once: its first entry speaks, with the
    // entries' probabilities added up in their order.
    speaks = 0;
#pragma unroll 1
    for (int k = tid, j = 0; k < p.K; k += nt, ++j) {
      const int at = rec.at[k];
      if (at < 0 || !s.holds(at)) continue;
      bool first = true;
      float q = 0.0f;
#pragma unroll 1
      for (int i = 0; i < p.K; ++i)
        if (rec.at[i] == at) {
          first &= i >= k;
          q += rec.q[i];
        }
      if (first) speaks |= 1u << j;
      rec.token_q[k] = q;
    }
    __syncthreads();
#pragma unroll 1
    for (int k = tid, j = 0; k < p.K; k += nt, ++j)
      if (speaks >> j & 1u) rec.q[k] = rec.token_q[k];
  }

  // The sums of 2^(z log2(e) / tau) over the record and over the rest, each relative
  // to a logit of its own: its maximum, and in the backward call the one that the
  // forward call's logarithm stands for.  The backward call adds them up again, since
  // a logarithm of about 20 in fp32 holds p to 1e-6 only; where the logarithms are so
  // large (or none) that their rounding is no small factor, it looks for the maxima.
  const float c2 = __fdiv_rn(kRowLog2e, p.tau);
  MaxSum in{-inf, 0.0f}, out{-inf, 0.0f};
  bool known = false;
  if (backward) {
    constexpr float kMost = 1048576.0f;  // 2^20: rounded by 2^-5
    const float l0 = p.stats[2ll * r], l1 = p.stats[2ll * r + 1];
    const float m0 = l0 * p.tau, m1 = l1 * p.tau;
    known = fabsf(l0) < kMost && fabsf(l1) < kMost && fabsf(m0) < 1e37f && fabsf(m1) < 1e37f;
    if (known) {
      in.m = m0;
      out.m = m1;
    }
  }
#pragma unroll 1
  for (int k = tid, j = 0; k < p.K; k += nt, ++j)
    if (speaks >> j & 1u) {
      const float z = rec.z[k];
      if (known)
        in.s += share_of(z, in.m, c2);
      else  // (z - z: NaN for an infinity)
        in = merge(in, MaxSum{z, z == -inf ? 0.0f : 1.0f + (z - z)}, c2);
    }
  load_slice<4>(s, [&](int v, const uint4& q) {
    float z[kVec];
    Row<T>::unpack(q, z);
    const uint32_t named = vector_bits<T>(bits, v);
    float m;
    if (named) {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (named >> e & 1u) z[e] = -inf;
      m = z[0];
#pragma unroll
      for (int e = 1; e < kVec; ++e) m = max_nan(m, z[e]);
    } else {
      m = vec_max(q, -inf, T());
    }
    if (!known && !(m <= out.m)) {  // a new maximum, or NaN
      out.s = out.m == -inf ? 0.0f : out.s * share_of(out.m, m, c2);
      out.m = m;
    }
    if (out.m != -inf) {
      float2 e2 = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) e2 = __fadd2_rn(e2, row_exp2_pair(z[e], z[e + 1], out.m, c2));
      out.s += e2.x + e2.y;
    }
  });
  c.begun();
  out = max_sum_of(cta_reduce(&sh, bits_of(out), MaxSumOp{c2}));
  in = max_sum_of(cta_reduce(&sh, bits_of(in), MaxSumOp{c2}, 1));
  {
    const unsigned long long mine[2] = {bits_of(out), bits_of(in)};
    const Parts parts = cluster_exchange(c, mine);
    out = max_sum_of(parts.of(0)[0]);
    in = max_sum_of(parts.of(1)[0]);
#pragma unroll 1
    for (int q = 1; q < c.ctas(); ++q) {
      out = merge(out, max_sum_of(parts.of(0)[q]), c2);
      in = merge(in, max_sum_of(parts.of(1)[q]), c2);
    }
  }
  const MaxSum all = merge(out, in, c2);
  const float ref = out.m == -inf ? 0.0f : out.m;
  if (!backward) {
    const float log_all = logf(all.s);
    float part = 0.0f;
#pragma unroll 1
    for (int k = tid; k < p.K; k += nt) {
      const int at = rec.at[k];
      if (at >= 0 && s.holds(at)) {
        const float q = expf(rec.logq[k]);
        if (q > 0.0f)
          part += q * (rec.logq[k] - (__fdiv_rn(rec.z[k] - all.m, p.tau) - log_all));
      }
    }
    part = cta_float(rec.scratch, part, add_op);
    if (tid == 0)
      c.store(reinterpret_cast<uint32_t*>(&rec.loss_part[c.rank()]), 0, __float_as_uint(part));
    c.sync();
    if (c.rank() == 0 && tid == 0) {
      float kl = 0.0f;
#pragma unroll 1
      for (int q = 0; q < c.ctas(); ++q) kl += rec.loss_part[q];
      const float log_rest = __fdiv_rn(out.m - all.m, p.tau) + (logf(out.s) - log_all);
      if (rest > 0.0f) kl += rest * (logf(rest) - log_rest);
      p.loss[r] = w * (p.tau * p.tau) * kl;
      p.stats[2ll * r] = __fdiv_rn(all.m, p.tau) + log_all;
      p.stats[2ll * r + 1] = __fdiv_rn(out.m, p.tau) + logf(out.s);
    }
  }
  if (!p.grad) return;

  const float up = (backward ? w * p.upstream[r] : w) * p.tau;
  // The student's probability of the rest as one class; of its gradient each
  // token has its part.  Where the class has no probability nothing is divided.
  const float p_rest = out.m == -inf ? 0.0f : out.s * share_of(out.m, all.m, c2) / all.s;
  const float coef = out.s > 0.0f || out.s != out.s ? up * (whole * p_rest - rest) / out.s : 0.0f;
  if (a_in == a_out) {
    for_slice<4, true>(s, [&](int v, const uint4& q) {
      float z[kVec];
      Row<T>::unpack(q, z);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const float2 g = __fmul2_rn(make_float2(coef, coef), row_exp2_pair(z[e], z[e + 1], ref, c2));
        z[e] = g.x;
        z[e + 1] = g.y;
      }
      if (v >= s.first && v < s.last) {
        __stcs(dst + v, Row<T>::pack(z));
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (s.holds(s.index(v) + e)) grow[s.index(v) + e] = Row<T>::from_float(z[e]);
      }
    });
  } else {
#pragma unroll 1
    for (int i = s.lo + tid; i < s.hi; i += nt) {
      const T z = kCluster ? reinterpret_cast<const T*>(s.kept)[i - s.index(0)] : row[i];
      grow[i] = Row<T>::from_float(coef * share_of(Row<T>::to_float(z), ref, c2));
    }
  }
  __syncthreads();  // the record's tokens come after
#pragma unroll 1
  for (int k = tid, j = 0; k < p.K; k += nt, ++j)
    if (speaks >> j & 1u) {
      const float pk = share_of(rec.z[k], all.m, c2) / all.s;
      grow[rec.at[k]] = Row<T>::from_float(up * (whole * pk - rec.q[k]));
    }
}

}  // namespace cai
