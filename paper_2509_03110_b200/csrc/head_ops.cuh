// head_ops.cuh -- scores of a classifier's head: log probability of the label, log-sum-exp, entropy and the top alternatives
// of every row of logits, and the gradient of a loss of the first and the third with respect to the logits.
#pragma once

#include "common.cuh"

namespace lsam {

constexpr float kLog2e = 1.4426950408889634f;  // log2 e, rounded
constexpr int kTopMax = 32;  // most alternatives a call returns (LSAM_TOP_MAX)

// 2^x, one instruction on the special-function unit (relative error below 2^-22; results below 2^-126 are flushed to 0)
__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Running statistics of a set of logits, held relative to its maximum m (NaN ignored) in units of log 2.  With k = kLog2e, B = fl(m k)
// and w = l k - B (one fused multiply-add):  s = sum 2^w,  t = sum 2^w w,  so that
//   logsumexp = m + (log2 s - (m k - B)) / k,   entropy = -sum p log p = (log2 s - t / s) / k.
// B is the reference itself, not an approximation of m k, and k's own rounding only scales the logits by 1 + 1e-8: an offset common to all
// logits costs no digits of the entropy or of a log probability.  Logits below kMasked are masks: they enter as kMasked, whose 2^w is 0
// beside any other (and (-inf) * 0 never arises); a set of nothing but masks has m = kMasked.  A NaN or +inf logit makes s NaN.
constexpr float kMasked = -1e30f;
struct RowStat { float m, s, t; };
__device__ inline float max_nan(float a, float b) {  // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ inline RowStat stat_empty() { return {kMasked, 0.f, 0.f}; }
__device__ inline void stat_rebase(RowStat& a, float m) {  // express a's sums relative to m >= a.m
  const float d = __fmul_rn(a.m, kLog2e) - __fmul_rn(m, kLog2e);  // the difference of the two references: never contracted
  const float f = ex2(d);
  a.t = f * fmaf(d, a.s, a.t);
  a.s *= f;
  a.m = m;
}
__device__ inline void stat_add(RowStat& a, float l) {  // one logit, masks and NaN included
  l = max_nan(l, kMasked);
  if (l > a.m) stat_rebase(a, l);
  const float w = fmaf(l, kLog2e, -(a.m * kLog2e));
  const float e = ex2(w);
  a.s += e;
  a.t = fmaf(e, w, a.t);
}
__device__ inline RowStat stat_merge(RowStat a, RowStat b) {
  const float m = fmaxf(a.m, b.m);
  stat_rebase(a, m);
  stat_rebase(b, m);
  return {m, a.s + b.s, a.t + b.t};
}
__device__ inline RowStat stat_shfl_xor(const RowStat& a, int d) {
  return {__shfl_xor_sync(~0u, a.m, d), __shfl_xor_sync(~0u, a.s, d), __shfl_xor_sync(~0u, a.t, d)};
}
struct RowScore { float B, ls, lse, ent; };
__device__ inline RowScore stat_finish(const RowStat& a) {
  if (a.m <= kMasked && a.s == a.s) return {0.f, 0.f, -INFINITY, 0.f};
  const float B = a.m * kLog2e, ls = log2f(a.s);
  return {B, ls, a.m + (ls - fmaf(a.m, kLog2e, -B)) / kLog2e, (ls - a.t / a.s) / kLog2e};
}
__device__ inline float score_logp(float l, const RowScore& r) { return l < kMasked ? -INFINITY : (fmaf(l, kLog2e, -r.B) - r.ls) / kLog2e; }

// Order of the alternatives: larger logit first, then the lower class.  One 64-bit key per element (0: not an alternative,
// i.e. a mask or NaN); -0 and +0 are one value.
__device__ inline uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float order_value(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ inline uint64_t order_key(float v, int32_t c) {
  return v >= kMasked ? ((uint64_t)order_bits(v) << 32) | (uint32_t)~c : 0ull;
}

// Logits of one call: element (k, r, c) at p[k * sk + r * sr + c * sc]; row index = k * rows + r.
template <typename T>
struct LogitView {
  const T* p;
  int64_t rows, sk, sr, sc;
  int32_t classes;
  __device__ inline const T* row(int64_t i) const { return p + (i / rows) * sk + (i % rows) * sr; }
};
struct ScoreOut {
  float *logp, *lse, *entropy, *top_logp;  // each nullable
  int32_t* top_idx;
  int32_t top_k;
};

// What a row that is left out (negative label) or has no finite logit returns beside its statistics.
__device__ inline void write_no_top(const ScoreOut& o, int64_t i, int from) {
  for (int j = from; j < o.top_k; ++j) {
    o.top_logp[i * o.top_k + j] = -INFINITY;
    o.top_idx[i * o.top_k + j] = -1;
  }
}

// One block per row: a strided pass for the statistics, then one pass per alternative (the best key below the previous one).
template <typename T>
__global__ void __launch_bounds__(256)
logprob_kernel(LogitView<T> v, const int32_t* __restrict__ labels, ScoreOut o) {
  __shared__ RowStat ws[8];
  __shared__ uint64_t wk[8];
  const int64_t i = blockIdx.x;
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  const int32_t y = labels ? labels[i] : 0;
  if (y < 0) {
    if (tid == 0) {
      if (o.logp) o.logp[i] = 0.f;
      if (o.lse) o.lse[i] = 0.f;
      if (o.entropy) o.entropy[i] = 0.f;
      write_no_top(o, i, 0);
    }
    return;
  }
  const T* row = v.row(i);
  RowStat a = stat_empty();
  for (int c = tid; c < v.classes; c += 256) stat_add(a, to_float(row[c * v.sc]));
  for (int d = 16; d > 0; d >>= 1) a = stat_merge(a, stat_shfl_xor(a, d));
  if (lane == 0) ws[w] = a;
  __syncthreads();
  a = ws[0];
  for (int q = 1; q < 8; ++q) a = stat_merge(a, ws[q]);
  const RowScore sc = stat_finish(a);
  if (tid == 0) {
    if (o.logp) o.logp[i] = y < v.classes ? score_logp(to_float(row[y * v.sc]), sc) : NAN;
    if (o.lse) o.lse[i] = sc.lse;
    if (o.entropy) o.entropy[i] = sc.ent;
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < o.top_k; ++j) {
    uint64_t best = 0;
    for (int c = tid; c < v.classes; c += 256) {
      const uint64_t k = order_key(to_float(row[c * v.sc]), c);
      if (k < last && k > best) best = k;
    }
    for (int d = 16; d > 0; d >>= 1) best = max(best, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)best, d));
    __syncthreads();
    if (lane == 0) wk[w] = best;
    __syncthreads();
    for (int q = 0; q < 8; ++q) best = max(best, wk[q]);
    if (best == 0) {
      if (tid == 0) write_no_top(o, i, j);
      break;
    }
    if (tid == 0) {
      o.top_logp[i * o.top_k + j] = score_logp(order_value((uint32_t)(best >> 32)), sc);
      o.top_idx[i * o.top_k + j] = (int32_t)~(uint32_t)best;
    }
    last = best;
  }
}

// Gradient of L(logp, entropy) of every row:  dl_c = a (1[c = y] - p_c) - b p_c (log p_c + H),  p_c = e^(l_c - lse),
// a = dL/dlogp, b = dL/dH (each nullable = 0).  Rows that are left out (y < 0) or hold nothing but masks (lse = -inf) get 0.
struct GradIn {
  const int32_t* labels;
  const float *lse, *entropy, *dlogp, *dentropy;
};
template <typename T>
struct GradOut { T* p; int64_t sk, sr, sc; };

template <typename T>
__global__ void __launch_bounds__(256)
logprob_grad_kernel(LogitView<T> v, GradIn g, GradOut<T> out) {
  const int64_t i = blockIdx.x;
  const int32_t y = g.labels ? g.labels[i] : v.classes - 1;
  const float lse = g.lse[i];
  T* dst = out.p + (i / v.rows) * out.sk + (i % v.rows) * out.sr;
  const bool none = y < 0 || lse < kMasked;
  const T* row = v.row(i);
  const float a = g.dlogp ? g.dlogp[i] : 0.f, b = g.dentropy ? g.dentropy[i] : 0.f, H = g.dentropy ? g.entropy[i] : 0.f;
  const float bad = y >= v.classes ? NAN : 0.f;
  for (int c = threadIdx.x; c < v.classes; c += 256) {
    float d = 0.f;
    if (!none) {
      const float u = max_nan(to_float(row[c * v.sc]), kMasked) - lse;
      const float p = ex2(u * kLog2e);
      d = a * ((c == y ? 1.f : 0.f) - p) - b * (p * (u + H)) + bad;
    }
    dst[c * out.sc] = from_float<T>(d);
  }
}

}  // namespace lsam
