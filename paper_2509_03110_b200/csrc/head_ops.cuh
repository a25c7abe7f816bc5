// head_ops.cuh -- scores of a classifier's head: log probability of the label, log-sum-exp, entropy and the top alternatives
// of every row of logits, and the gradient of a loss of the first and the third with respect to the logits.
#pragma once

#include <type_traits>

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

// Running statistics of a set of logits, held relative to its maximum m (NaN ignored) in units of log 2.  With k = kLog2e and w = (l - m) k:
//   s = sum 2^w,  t = sum 2^w w,  logsumexp = m + log2 s / k,   entropy = -sum p log p = (log2 s - t / s) / k.
// The difference l - m comes first: near the maximum it is exact, so an offset common to all logits, however large, costs no digits of the entropy
// or of a log probability (l k - m k in one multiply-add would be off by the rounding of m k: 2^85 at m = -1e9, a usual mask).
// Logits at or below kMasked are masks: they enter as kMasked, whose 2^w is 0 beside any other (and (-inf) * 0 never arises); a set of nothing but
// masks has m = kMasked.  A NaN or +inf logit makes s NaN.
constexpr float kMasked = -1e30f;
__device__ inline float above_masked() { return __uint_as_float(__float_as_uint(kMasked) - 1u); }  // the least fp32 number above it
struct RowStat { float m, s, t; };
__device__ inline float max_nan(float a, float b) {  // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ inline RowStat stat_empty() { return {kMasked, 0.f, 0.f}; }
__device__ inline void stat_rebase(RowStat& a, float m) {  // express a's sums relative to m >= a.m
  const float d = fmaxf((a.m - m) * kLog2e, -1000.f);  // 2^-1000 is 0, and d s stays finite
  const float f = ex2(d);
  a.t = f * fmaf(d, a.s, a.t);
  a.s *= f;
  a.m = m;
}
__device__ inline void stat_add(RowStat& a, float l) {  // one logit, masks and NaN included
  l = max_nan(l, kMasked);
  if (l > a.m) stat_rebase(a, l);
  const float w = (l - a.m) * kLog2e;
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
__device__ inline float warp_max_f(float v) {  // NaN ignored
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(v));
  return y;
}
// The statistics of a warp's 32 sets, in every lane: one rebase to the common maximum, then two sums in the order of the xor tree.
__device__ inline RowStat warp_stat(RowStat a) {
  stat_rebase(a, warp_max_f(a.m));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, d);
    a.t += __shfl_xor_sync(~0u, a.t, d);
  }
  return a;
}
struct RowScore { float m, ls, lse, ent; };  // ls = lse - m
__device__ inline RowScore stat_finish(const RowStat& a) {
  if (a.m <= kMasked && a.s == a.s) return {0.f, 0.f, -INFINITY, 0.f};
  const float b = log2f(a.s), ls = b / kLog2e;
  return {a.m, ls, a.m + ls, (b - a.t / a.s) / kLog2e};
}
// lse + lse_low(r) is m + ls to twice the digits (the error of the sum m + ls, exact in six additions)
__device__ inline float lse_low(const RowScore& r) {
  const float s = r.m + r.ls, b = s - r.m;
  return (r.m - (s - b)) + (r.ls - b);
}
__device__ inline float score_logp(float l, const RowScore& r) { return l <= kMasked ? -INFINITY : (l - r.m) - r.ls; }

// Order of the alternatives: larger logit first, then the lower class.  One 64-bit key per element (0: not an alternative,
// i.e. a mask or NaN); -0 and +0 are one value.
__device__ inline uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float order_value(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ inline uint64_t order_key(float v, int32_t c) {
  return v > kMasked ? ((uint64_t)order_bits(v) << 32) | (uint32_t)~c : 0ull;
}

// Logits of one call: element (k, r, c) at p[k * sk + r * sr + c * sc]; row index i = k * rows + r < 2^31.
template <typename T>
struct LogitView {
  const T* p;
  int64_t rows, sk, sr, sc;
  int32_t classes;
  FastDiv by_rows;
  __device__ inline const T* row(uint32_t i) const {
    uint32_t r;
    const uint32_t k = by_rows.div(i, r);
    return p + k * sk + r * sr;
  }
};
struct ScoreOut {
  float *logp, *lse, *entropy, *top_logp;  // each nullable
  int32_t* top_idx;
  int32_t top_k;
  float* lse_low;  // nullable: what the rounding of lse to 32 bits leaves out
};

// What a row that is left out (negative label) or has no finite logit returns beside its statistics.
__device__ inline void write_no_top(const ScoreOut& o, int64_t i, int from) {
  for (int j = from; j < o.top_k; ++j) {
    o.top_logp[i * o.top_k + j] = -INFINITY;
    o.top_idx[i * o.top_k + j] = -1;
  }
}

// ---- 16-byte vectors of logits
template <typename T> __host__ __device__ constexpr int vec_n() { return 16 / (int)sizeof(T); }
template <typename T> __device__ inline void vec_unpack(const uint4& q, float (&f)[16 / sizeof(T)]);
template <> __device__ inline void vec_unpack<float>(const uint4& q, float (&f)[4]) {
  f[0] = __uint_as_float(q.x); f[1] = __uint_as_float(q.y); f[2] = __uint_as_float(q.z); f[3] = __uint_as_float(q.w);
}
template <> __device__ inline void vec_unpack<bf16>(const uint4& q, float (&f)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(w[j] << 16); f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
template <> __device__ inline void vec_unpack<fp16>(const uint4& q, float (&f)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
    f[2 * j] = p.x; f[2 * j + 1] = p.y;
  }
}
// two fp32 operations per instruction
__device__ inline uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ inline void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ inline uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ inline uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Statistics of N logits that are already cut at kMasked, mx their maximum (NaN ignored).
template <int N>
__device__ inline void stat_add_all(RowStat& a, const float (&l)[N], float mx) {
  static_assert(N % 2 == 0, "pairs");
  if (mx > a.m) stat_rebase(a, mx);
  const uint64_t k2 = pack2(kLog2e, kLog2e), m2 = pack2(-a.m, -a.m);
  uint64_t s2 = 0, t2 = 0;
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    const uint64_t w2 = mul2(add2(pack2(l[j], l[j + 1]), m2), k2);
    float w0, w1;
    unpack2(w2, w0, w1);
    const uint64_t e2 = pack2(ex2(w0), ex2(w1));
    s2 = add2(s2, e2);
    t2 = fma2(e2, w2, t2);
  }
  float x, y;
  unpack2(s2, x, y);
  a.s += x + y;
  unpack2(t2, x, y);
  a.t += x + y;
}
// Cuts U vectors at kMasked and adds them; returns their maximum.
template <typename T, int U>
__device__ inline float stat_add_vecs(RowStat& a, uint4 (&q)[U]) {
  constexpr int N = vec_n<T>();
  float mx = kMasked, l[U * N];
  if constexpr (sizeof(T) == 2) {
    // 16-bit logits are compared in pairs; until their exponentials they stay packed (held as floats, a step of fp16 would not leave room for five
    // blocks).  bf16 is cut in pairs too, at the bf16 next below kMasked; fp16 has no such number and is cut after the conversion.
    constexpr bool BF = std::is_same<T, bf16>::value;
    uint32_t m2 = BF ? 0xf14af14au : 0xfc00fc00u;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&q[u]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (BF) {
          asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w[j]) : "r"(w[j]), "r"(0xf14af14au));
          asm("max.bf16x2 %0, %1, %2;" : "=r"(m2) : "r"(m2), "r"(w[j]));
        } else {
          asm("max.f16x2 %0, %1, %2;" : "=r"(m2) : "r"(m2), "r"(w[j]));
        }
      }
    }
    float top[2];
    if (BF) {
      top[0] = __uint_as_float(m2 << 16); top[1] = __uint_as_float(m2 & 0xffff0000u);
    } else {
      const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&m2));
      top[0] = t.x; top[1] = t.y;
    }
    mx = fmaxf(mx, fmaxf(top[0], top[1]));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      vec_unpack<T>(q[u], f);
#pragma unroll
      for (int j = 0; j < N; ++j) l[u * N + j] = BF ? f[j] : max_nan(f[j], kMasked);
    }
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      vec_unpack<T>(q[u], f);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        l[u * N + j] = max_nan(f[j], kMasked);
        mx = fmaxf(mx, l[u * N + j]);
      }
    }
  }
  stat_add_all(a, l, mx);
  return mx;
}

__device__ inline void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename V>
__device__ inline const V* cluster_map(const V* p, uint32_t rank) {  // the same shared variable of another block of the cluster
  uint64_t r;
  asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<const V*>(r);
}

// Which elements of a row a thread owns.  The row is [head scalars][16-byte vectors][tail scalars]; thread g of G owns scalars and vectors
// g, g + G, ... of each part.  A row without unit stride is all head.
template <typename T>
struct RowParts {
  const T* row;
  int64_t sc;
  int32_t head, nvec, tail0, classes;
  __device__ inline RowParts(const T* r, int64_t stride, int32_t C) : row(r), sc(stride), classes(C) {
    if (stride != 1) { head = C; nvec = 0; tail0 = C; return; }
    const int32_t off = (int32_t)((16 - (reinterpret_cast<uintptr_t>(r) & 15)) & 15) / (int32_t)sizeof(T);
    head = off < C ? off : C;
    nvec = (C - head) / vec_n<T>();
    tail0 = head + nvec * vec_n<T>();
  }
  __device__ inline float at(int64_t c) const { return to_float(row[c * sc]); }
  __device__ inline uint4 vec(int32_t v) const { return __ldg(reinterpret_cast<const uint4*>(row + head) + v); }
  // f(value, class) for every element >= thr that thread g of G owns; `lanes` threads take its vectors in turn
  template <class F>
  __device__ inline void each_of(int g, int G, int lane, int lanes, float thr, F&& f) const {
    auto see = [&](float l, int32_t c) {
      if (l >= thr) f(l, c);
    };
    if (head > 0)
      for (int64_t c = g + (int64_t)lane * G; c < head; c += (int64_t)lanes * G) see(at(c), (int32_t)c);
    const int32_t step = lanes * G;
#pragma unroll 2
    for (int32_t v = g + lane * G; v < nvec; v += step) {
      float l[vec_n<T>()];
      vec_unpack<T>(vec(v), l);
      float mx = l[0];
#pragma unroll
      for (int j = 1; j < vec_n<T>(); ++j) mx = fmaxf(mx, l[j]);
      if (mx >= thr) {
#pragma unroll
        for (int j = 0; j < vec_n<T>(); ++j) see(l[j], head + v * vec_n<T>() + j);
      }
    }
    const int64_t c = (int64_t)tail0 + g;  // the tail is shorter than a vector
    if (lane == 0 && c < classes) see(at(c), (int32_t)c);
  }
};

// k-th largest (1 <= k <= 32) of the values of a warp's lanes.  Small k: the maximum is taken and one lane that holds it leaves, k times; else the
// least value that fewer than k others exceed (31 independent exchanges instead of k dependent steps).
__device__ inline float warp_kth(float v, int k) {
  float t;
  if (k <= 4) {
    for (int j = 0;; ++j) {
      t = warp_max_f(v);
      if (j == k - 1) return t;
      const uint32_t who = __ballot_sync(~0u, v == t);
      if ((threadIdx.x & 31) == __ffs(who) - 1) v = -INFINITY;
    }
  }
  int above = 0;
#pragma unroll
  for (int d = 1; d < 32; ++d) above += __shfl_xor_sync(~0u, v, d) > v;
  const float low = above < k ? v : INFINITY;
  asm("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(t) : "f"(low));
  return t;
}

constexpr int kTopList = 512;  // candidates a block keeps
// What a thread knows of its own elements: the first vector of the step that holds its maximum (-1: a scalar does) and the maximum of all others.
struct StepMax {
  int32_t step = -1;
  float second = kMasked;
  __device__ inline void see(float before, float mx, int32_t q) {
    if (mx > before) { second = before; step = q; }
    else second = fmaxf(second, mx);
  }
};
constexpr int kStep = 4;  // vectors a thread takes per step
template <int NT>
struct TopShared {
  float maxima[NT], second[NT];
  int32_t step[NT];
  int owners[NT];
  uint64_t above[kTopList], equal[kTopList];  // keys of elements above / at the threshold
  uint64_t best[kTopMax];
  int n_own, n_above, n_equal;
  float thr;
};

// The k best keys of the elements that the NT threads of a block own -> sh.best in order (0: none), valid after the call.  vm = the
// caller's own maximum (cut at kMasked, NaN ignored).  T = the k-th largest of 32 maxima, each over NT / 32 threads: at least k elements are >= T, so
// the k best are, and on rows without order about 32 log(32 / (32 - k)) are (9 for k = 8, 31 for k = 20).  Only threads whose maximum reaches T
// ("owners") have elements read again, the step that holds the maximum (64 bytes), or all of them where another step reaches T too; what
// passes T is ranked by counting.  (A row of 256 KB has partly left L2 by then: reading all of an owner's elements again cost 17 us per 2048 rows.)
//   More than kTopList elements at T (tied rows): the lowest classes are picked in order by one warp, which stops at the k-th.
//   More than kTopList above T: k passes over the owners' elements.
template <typename T, int NT>
__device__ void block_top(const RowParts<T>& rp, int g0, int G, float vm, const StepMax& sm, int k, TopShared<NT>& sh) {
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  constexpr int NW = NT / 32, LIST = kTopList, U = kStep;
  sh.maxima[tid] = vm;
  sh.second[tid] = sm.second;
  sh.step[tid] = sm.step;
  __syncthreads();
  if (w == 0) {
    float m[NW];
#pragma unroll
    for (int q = 0; q < NW; ++q) m[q] = sh.maxima[q * 32 + lane];
    float mine = m[0];
#pragma unroll
    for (int q = 1; q < NW; ++q) mine = fmaxf(mine, m[q]);
    const float t = warp_kth(mine, k);
    int n = 0;  // owners in lane order
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      const bool own = m[q] >= t && m[q] > kMasked;
      const uint32_t who = __ballot_sync(~0u, own);
      if (own) sh.owners[n + __popc(who & ((1u << lane) - 1u))] = q * 32 + lane;
      n += __popc(who);
    }
    if (lane == 0) { sh.thr = t; sh.n_own = n; sh.n_above = sh.n_equal = 0; }
    sh.best[lane] = 0;
  }
  __syncthreads();
  const float thr = sh.thr;
  const int n_own = sh.n_own;
  const bool owner = vm >= thr && vm > kMasked;
  // all elements of the owners that `which` names: few owners, a warp takes one at a time, its lanes read the owner's vectors side by side;
  // many (tied rows), every owner reads its own
  auto each_candidate = [&](auto&& f, auto&& which) {
    if (n_own <= 8 * NW) {
      for (int q = w; q < n_own; q += NW)
        if (which(sh.owners[q])) rp.each_of(g0 + sh.owners[q], G, lane, 32, thr, f);
    } else if (owner && which(tid)) {
      rp.each_of(g0 + tid, G, 0, 1, thr, f);
    }
  };
  auto offer = [&](float l, int32_t c) {
    if (l > thr) {
      const int at = atomicAdd(&sh.n_above, 1);
      if (at < LIST) sh.above[at] = order_key(l, c);
    } else if (l == thr && l > kMasked) {
      const int at = atomicAdd(&sh.n_equal, 1);
      if (at < LIST) sh.equal[at] = order_key(l, c);
    }
  };
  for (int e = tid; e < n_own * U; e += NT) {
    const int own = sh.owners[e / U], u = e % U;
    const int32_t q = sh.step[own];
    if (q >= 0 && sh.second[own] < thr && (u == 0 || q + (U - 1) * G < rp.nvec)) {  // the row's last vectors are steps of one
      const int32_t v = q + u * G;
      float l[vec_n<T>()];
      vec_unpack<T>(rp.vec(v), l);
#pragma unroll
      for (int j = 0; j < vec_n<T>(); ++j)
        if (l[j] >= thr) offer(l[j], rp.head + v * vec_n<T>() + j);
    }
  }
  each_candidate(offer, [&](int own) { return sh.step[own] < 0 || sh.second[own] >= thr; });
  __syncthreads();
  const int na = sh.n_above, ne = sh.n_equal;
  if (na > LIST) {
    uint64_t last = ~0ull;
    for (int j = 0; j < k; ++j) {
      uint64_t best = 0;
      auto see = [&](float l, int32_t c) {
        const uint64_t key = order_key(l, c);
        if (key < last && key > best) best = key;
      };
      each_candidate(see, [](int) { return true; });
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) best = max(best, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)best, d));
      __syncthreads();
      if (lane == 0) sh.equal[w] = best;
      __syncthreads();
      for (int q = 0; q < NW; ++q) best = max(best, sh.equal[q]);
      if (tid == 0) sh.best[j] = best;
      last = best;  // 0: nothing is left
    }
    __syncthreads();
    return;
  }
  for (int q = tid; q < na; q += NT) {
    const uint64_t key = sh.above[q];
    int r = 0;
    for (int p = 0; p < na; ++p) r += sh.above[p] > key;
    if (r < k) sh.best[r] = key;
  }
  if (na < k && ne <= LIST) {
    for (int q = tid; q < ne; q += NT) {
      const uint64_t key = sh.equal[q];
      int r = na;
      for (int p = 0; p < ne; ++p) r += sh.equal[p] > key;
      if (r < k) sh.best[r] = key;
    }
  } else if (na < k && w == 0) {
    int have = na;  // the lowest classes at T, in order
    auto take = [&](uint32_t mask, int32_t c0) {  // this lane's elements c0 + bit, lanes ascending
      int incl = __popc(mask);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, incl, d);
        if (lane >= d) incl += o;
      }
      int at = have + incl - __popc(mask);
      for (; mask && at < k; mask &= mask - 1) sh.best[at++] = order_key(thr, c0 + __ffs(mask) - 1);
      have += __shfl_sync(~0u, incl, 31);
    };
    for (int64_t j = 0; j < rp.head && have < k; j += G)
      for (int t = 0; t < NT && have < k; t += 32) {
        const int64_t c = j + g0 + t + lane;
        take(c < rp.head && rp.at(c) == thr, (int32_t)c);
      }
    for (int64_t j = 0; j < rp.nvec && have < k; j += G)
      for (int t = 0; t < NT && have < k; t += 32) {
        const int64_t v = j + g0 + t + lane;
        uint32_t mask = 0;
        if (v < rp.nvec) {
          float l[vec_n<T>()];
          vec_unpack<T>(rp.vec((int32_t)v), l);
#pragma unroll
          for (int e = 0; e < vec_n<T>(); ++e) mask |= (l[e] == thr ? 1u : 0u) << e;
        }
        take(mask, rp.head + (int32_t)v * vec_n<T>());
      }
    const int64_t c = (int64_t)rp.tail0 + g0 + lane;  // the tail is shorter than a vector
    if (have < k) take(c < rp.classes && rp.at(c) == thr, (int32_t)c);
  }
  __syncthreads();
}

__device__ inline void write_left_out(const ScoreOut& o, int64_t i) {
  if (o.logp) o.logp[i] = 0.f;
  if (o.lse) o.lse[i] = 0.f;
  if (o.entropy) o.entropy[i] = 0.f;
  if (o.lse_low) o.lse_low[i] = 0.f;
  write_no_top(o, i, 0);
}
__device__ inline void write_scores(const ScoreOut& o, int64_t i, const RowScore& sc, int32_t y, int32_t classes, float at_label) {
  if (o.logp) o.logp[i] = y < classes ? score_logp(at_label, sc) : NAN;
  if (o.lse) o.lse[i] = sc.lse;
  if (o.entropy) o.entropy[i] = sc.ent;
  if (o.lse_low) o.lse_low[i] = lse_low(sc);
}
__device__ inline void write_top(const ScoreOut& o, int64_t i, int j, uint64_t key, const RowScore& sc) {
  o.top_logp[i * o.top_k + j] = key ? score_logp(order_value((uint32_t)(key >> 32)), sc) : -INFINITY;
  o.top_idx[i * o.top_k + j] = key ? (int32_t)~(uint32_t)key : -1;
}

// The alternatives of a row whose 32 x n elements sit in the registers of one warp: the k best keys -> best (shared memory, kTopMax), `list` its candidate
// list.  thr: at least k elements reach it.  key(j): the caller's j-th key (0: no alternative).
template <int N, class F>
__device__ inline void warp_top(float thr, const float (&l)[N], int k, uint64_t* list, int list_n, int* count, uint64_t* best, F&& class_of) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) *count = 0;
  best[lane] = 0;
  const float least = fmaxf(thr, above_masked());
  __syncwarp();
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (l[j] >= least) {
      const int at = atomicAdd(count, 1);
      if (at < list_n) list[at] = order_key(l[j], class_of(j));
    }
  __syncwarp();
  const int n = *count;
  if (n <= list_n) {
    for (int q = lane; q < n; q += 32) {
      const uint64_t key = list[q];
      int r = 0;
      for (int z = 0; z < n; ++z) r += list[z] > key;
      if (r < k) best[r] = key;
    }
  } else {
    // more candidates than the list holds (ties): the best key below the previous one, k times
    uint64_t last = ~0ull;
    for (int j = 0; j < k; ++j) {
      uint64_t b = 0;
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const uint64_t key = order_key(l[q], class_of(q));
        if (key < last && key > b) b = key;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) b = max(b, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)b, d));
      if (lane == 0) best[j] = b;
      last = b;
    }
  }
  __syncwarp();
}

// Rows of at most 1024 classes: a warp per row, 32 logits a lane in registers, so that the maximum is known before the first exponential and the
// alternatives cost no second read.  VEC: every row starts on a 16-byte boundary.
constexpr int kWarpClasses = 1024, kWarpList = 64;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
logprob_warp_kernel(LogitView<T> v, const int32_t* __restrict__ labels, ScoreOut o, uint32_t total) {
  __shared__ uint64_t list[8][kWarpList], best[8][kTopMax];
  __shared__ int count[8];
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t i = blockIdx.x * 8 + w;
  if (i >= total) return;
  const int32_t y = labels ? labels[i] : 0;
  if (y < 0) {
    if (lane == 0) write_left_out(o, i);
    return;
  }
  const T* row = v.row(i);
  const float at_label = lane == 0 && o.logp && y < v.classes ? to_float(row[y * v.sc]) : NAN;
  constexpr int N = vec_n<T>();
  float l[32];
  if (VEC) {
    uint4 x[32 / N];
    const int nvec = v.classes / N;
#pragma unroll
    for (int j = 0; j < 32 / N; ++j)
      if (j * 32 + lane < nvec) x[j] = __ldg(reinterpret_cast<const uint4*>(row) + j * 32 + lane);
#pragma unroll
    for (int j = 0; j < 32 / N; ++j) {
      float f[N];
      if (j * 32 + lane < nvec) {
        vec_unpack<T>(x[j], f);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int c = (j * 32 + lane) * N + e;
          f[e] = c < v.classes ? to_float(row[c]) : -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) l[j * N + e] = f[e];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const int c = j * 32 + lane;
      l[j] = c < v.classes ? to_float(row[c * v.sc]) : -INFINITY;
    }
  }
  float mx = kMasked;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    l[j] = max_nan(l[j], kMasked);
    mx = fmaxf(mx, l[j]);
  }
  RowStat a = {warp_max_f(mx), 0.f, 0.f};
  stat_add_all(a, l, a.m);
  a = warp_stat(a);
  const RowScore sc = stat_finish(a);
  if (lane == 0) write_scores(o, i, sc, y, v.classes, at_label);
  if (o.top_k == 0) return;
  warp_top(warp_kth(mx, o.top_k), l, o.top_k, list[w], kWarpList, &count[w], best[w], [&](int j) { return VEC ? (j / N * 32 + lane) * N + j % N : j * 32 + lane; });
  if (lane < o.top_k) write_top(o, i, lane, best[w][lane], sc);
}

// Blocks per SM a form is compiled for.  Measured (us, without / with 8 alternatives): 2048 x 131072 bf16: 256 threads x 5 blocks 89 / 99, x 6 (spilling) 99 /
// 110, 512 threads x 3 94 / 107;  4096 x 32768 bf16: 256 x 5 49 / 65, 128 threads x 10 51 / 64, 512 x 3 58 / 82;  8192 x 8192 fp32: 128 x 10 43 / 57,
// 256 x 5 43 / 70.  A loop that kept the next step's loads in flight gained nothing over the blocks it cost.
template <int NT, int CS> __host__ __device__ constexpr int row_blocks() { return CS > 1 ? 4 : NT == 256 ? 5 : 10; }

// Rows of contiguous classes (or of any stride, one element at a time): NT threads of CS blocks (a cluster) per row, one pass.  A thread keeps the
// statistics of the vectors it owns in registers, a step of them at a time; nothing is exchanged until the row ends.
template <typename T, int NT, int CS>
__global__ void __launch_bounds__(NT, row_blocks<NT, CS>())
logprob_row_kernel(LogitView<T> v, const int32_t* __restrict__ labels, ScoreOut o) {
  constexpr int NW = NT / 32, U = kStep, G = NT * CS;
  __shared__ RowStat ws[NW], cta;
  __shared__ TopShared<NT> sh;
  const uint32_t i = blockIdx.x / CS;
  const int part = CS > 1 ? (int)(blockIdx.x % CS) : 0;
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g0 = part * NT, g = g0 + tid;
  const int32_t y = labels ? labels[i] : 0;
  if (y < 0) {  // the same for every block of the cluster
    if (g == 0) write_left_out(o, i);
    return;
  }
  const RowParts<T> rp(v.row(i), v.sc, v.classes);
  const float at_label = g == 0 && o.logp && y < v.classes ? rp.at(y) : NAN;  // asked for now, needed when the row ends
  RowStat a = stat_empty();
  for (int64_t c = g; c < rp.head; c += G) stat_add(a, rp.at(c));
  if ((int64_t)rp.tail0 + g < rp.classes) stat_add(a, rp.at(rp.tail0 + g));
  StepMax sm;
  int32_t q = g;
  for (; q + (U - 1) * G < rp.nvec; q += U * G) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = rp.vec(q + u * G);
    const float before = a.m;
    sm.see(before, stat_add_vecs<T, U>(a, x), q);
  }
  for (; q < rp.nvec; q += G) {
    uint4 x[1] = {rp.vec(q)};
    const float before = a.m;
    sm.see(before, stat_add_vecs<T, 1>(a, x), q);
  }
  const float vm = a.m;
  a = warp_stat(a);
  if (lane == 0) ws[w] = a;
  if (o.top_k == 0) __syncthreads();  // else block_top's barriers order this
  else block_top<T, NT>(rp, g0, G, vm, sm, o.top_k, sh);
  if (w == 0) a = warp_stat(lane < NW ? ws[lane] : stat_empty());  // from here on only warp 0 holds the row's statistics
  if (CS > 1) {
    if (tid == 0) cta = a;
    cluster_sync();
    if (part == 0) {
      if (w == 0) a = warp_stat(lane < CS ? *cluster_map(&cta, lane) : stat_empty());
      if (o.top_k > 0) {
        // rank the CS * k keys of the blocks: all into this block's list first
        const int n = CS * o.top_k;
        for (int p = tid; p < n; p += NT) sh.above[p] = cluster_map(sh.best, p / o.top_k)[p % o.top_k];
        if (tid < kTopMax) sh.equal[tid] = 0;
        __syncthreads();
        for (int p = tid; p < n; p += NT) {
          const uint64_t key = sh.above[p];
          int r = 0;
          for (int z = 0; z < n; ++z) r += sh.above[z] > key;
          if (key && r < o.top_k) sh.equal[r] = key;
        }
        __syncthreads();
      }
    }
    cluster_sync();  // no block leaves while its shared memory is read
    if (part != 0) return;
  }
  if (w != 0) return;
  const RowScore sc = stat_finish(a);
  if (tid == 0) write_scores(o, i, sc, y, v.classes, at_label);
  if (tid < o.top_k) write_top(o, i, tid, CS > 1 ? sh.equal[tid] : sh.best[tid], sc);
}

// Logits with the sample index contiguous: R rows (32 bytes' worth) x 32 groups of classes per block, group y owns classes y, y + 32, ...; a warp
// reads whole 32-byte sectors.  A chunk of 32 x kFeatN classes is loaded into registers in one go, and stays there for the alternatives when it is the whole row.
constexpr int kFeatG = 32, kFeatN = 32, kFeatList = 48;
template <typename T> __host__ __device__ constexpr int feat_rows() { return 32 / (int)sizeof(T); }
template <typename T>
__global__ void __launch_bounds__(feat_rows<T>() * kFeatG, 1024 / (feat_rows<T>() * kFeatG))
logprob_feature_kernel(LogitView<T> v, const int32_t* __restrict__ labels, ScoreOut o, uint32_t row_blocks) {
  constexpr int kFeatR = feat_rows<T>();
  __shared__ float red[3][kFeatR][kFeatG + 1];
  __shared__ uint64_t list[kFeatR][kFeatList];
  __shared__ uint64_t best[kFeatR][kTopMax];
  __shared__ float thr_s[kFeatR];
  __shared__ int count[kFeatR];
  const int x = threadIdx.x % kFeatR, y = threadIdx.x / kFeatR;
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t k = blockIdx.x / row_blocks;
  const int64_t r0 = (int64_t)(blockIdx.x % row_blocks) * kFeatR, r = r0 + x, i = k * v.rows + r;
  const bool in = r < v.rows;
  const int32_t lab = in && labels ? labels[i] : 0;
  const bool live = in && lab >= 0;
  const T* p = v.p + k * v.sk + (live ? r : 0) * v.sr;
  const int64_t step = kFeatG * v.sc;
  RowStat a = stat_empty();
  float l[kFeatN];
  for (int64_t c0 = y; c0 < v.classes || c0 == y; c0 += kFeatG * kFeatN) {
    float mx = kMasked;
    const int n = live ? (int)min((int64_t)kFeatN, (v.classes - c0 + kFeatG - 1) / kFeatG) : 0;  // this thread's classes of the chunk
    const T* q = p + c0 * v.sc;
#pragma unroll
    for (int j = 0; j < kFeatN; ++j, q += step) l[j] = j < n ? to_float(*q) : -INFINITY;
#pragma unroll
    for (int j = 0; j < kFeatN; ++j) {
      l[j] = max_nan(l[j], kMasked);
      mx = fmaxf(mx, l[j]);
    }
    stat_add_all(a, l, mx);
  }
  // warp w ends row w; its label's logit is asked for before the block meets
  const int64_t rw = r0 + w, iw = k * v.rows + rw;
  const bool row_in = rw < v.rows;
  const int32_t yw = row_in && labels ? labels[iw] : 0;
  const T* pw = v.p + k * v.sk + (row_in ? rw : 0) * v.sr;
  const float at_label = lane == 0 && row_in && o.logp && yw >= 0 && yw < v.classes ? to_float(pw[(int64_t)yw * v.sc]) : NAN;
  const float vm = a.m;
  red[0][x][y] = a.m; red[1][x][y] = a.s; red[2][x][y] = a.t;
  if (threadIdx.x < kFeatR) count[threadIdx.x] = 0;
  __syncthreads();
  // warp w joins row w over its 32 groups; the threshold of the row is the k-th largest of the groups' maxima
  a = {red[0][w][lane], red[1][w][lane], red[2][w][lane]};
  if (o.top_k > 0) {
    const float t = warp_kth(a.m, o.top_k);
    if (lane == 0) thr_s[w] = t;
    best[w][lane] = 0;
  }
  a = warp_stat(a);
  const RowScore sc = stat_finish(a);
  if (lane == 0 && row_in) {
    if (yw < 0) write_left_out(o, iw);
    else write_scores(o, iw, sc, yw, v.classes, at_label);
  }
  if (o.top_k == 0) return;
  __syncthreads();
  const float least = fmaxf(thr_s[x], above_masked());
  auto offer = [&](float val, int64_t c) {
    if (val >= least) {
      const int at = atomicAdd(&count[x], 1);
      if (at < kFeatList) list[x][at] = order_key(val, (int32_t)c);
    }
  };
  if (live && vm >= least) {
    if (v.classes <= kFeatG * kFeatN) {
#pragma unroll
      for (int j = 0; j < kFeatN; ++j) offer(l[j], y + kFeatG * j);
    } else {
      for (int64_t c = y; c < v.classes; c += kFeatG) offer(to_float(p[c * v.sc]), c);
    }
  }
  __syncthreads();
  if (!row_in || yw < 0) return;
  const int n = count[w];
  if (n <= kFeatList) {
    for (int q = lane; q < n; q += 32) {
      const uint64_t key = list[w][q];
      int rank = 0;
      for (int z = 0; z < n; ++z) rank += list[w][z] > key;
      if (rank < o.top_k) best[w][rank] = key;
    }
  } else {
    // more candidates than the list holds (ties): one pass of the warp per alternative
    uint64_t last = ~0ull;
    for (int j = 0; j < o.top_k; ++j) {
      uint64_t b = 0;
      for (int64_t c = lane; c < v.classes; c += 32) {
        const uint64_t key = order_key(to_float(pw[c * v.sc]), (int32_t)c);
        if (key < last && key > b) b = key;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) b = max(b, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)b, d));
      if (lane == 0) best[w][j] = b;
      last = b;
    }
  }
  __syncwarp();
  if (lane < o.top_k) write_top(o, iw, lane, best[w][lane], sc);
}

// Many rows of few classes: a thread per row, 16 logits at a time; an alternative costs one more walk over the row, which is in L1 or L2.
template <typename T>
__global__ void __launch_bounds__(128)
logprob_thread_kernel(LogitView<T> v, const int32_t* __restrict__ labels, ScoreOut o, uint32_t total) {
  const uint32_t i = blockIdx.x * 128 + threadIdx.x;
  if (i >= total) return;
  const int32_t y = labels ? labels[i] : 0;
  if (y < 0) {
    write_left_out(o, i);
    return;
  }
  const T* row = v.row(i);
  RowStat a = stat_empty();
  for (int32_t c0 = 0; c0 < v.classes; c0 += 16) {
    float l[16], mx = kMasked;
    const T* p = row + c0 * v.sc;
#pragma unroll
    for (int j = 0; j < 16; ++j, p += v.sc) l[j] = c0 + j < v.classes ? to_float(*p) : -INFINITY;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      l[j] = max_nan(l[j], kMasked);
      mx = fmaxf(mx, l[j]);
    }
    stat_add_all(a, l, mx);
  }
  const RowScore sc = stat_finish(a);
  write_scores(o, i, sc, y, v.classes, o.logp && y < v.classes ? to_float(row[y * v.sc]) : NAN);
  float last = INFINITY;  // the previous alternative: the next one is the first largest behind it in (value, class) order
  int32_t last_c = -1;
  for (int k = 0; k < o.top_k; ++k) {
    float best = kMasked;
    int32_t best_c = -1;
    if (k == 0 || last_c >= 0) {
      for (int32_t c0 = 0; c0 < v.classes; c0 += 16) {
        float l[16];
        const T* p = row + c0 * v.sc;
#pragma unroll
        for (int j = 0; j < 16; ++j, p += v.sc) l[j] = c0 + j < v.classes ? to_float(*p) : -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (l[j] > best && (l[j] < last || (l[j] == last && c0 + j > last_c))) { best = l[j]; best_c = c0 + j; }
      }
    }
    o.top_logp[(int64_t)i * o.top_k + k] = best_c >= 0 ? score_logp(best, sc) : -INFINITY;
    o.top_idx[(int64_t)i * o.top_k + k] = best_c;
    last = best;
    last_c = best_c;
  }
}

// Gradient of L(logp, entropy) of every row:  dl_c = a (1[c = y] - p_c) - b p_c (log p_c + H),  p_c = e^(l_c - lse),
// a = dL/dlogp, b = dL/dH (each nullable = 0).  Rows that are left out (y < 0) or hold nothing but masks (lse = -inf) get 0.
// With u = l - lse it is p (c0 + c1 u), c0 = -(a + b H), c1 = -b, plus a at the label: one read, one write, two multiply-adds and one exponential
// per element, bound by the bytes.
// lse rounded to 32 bits is off by up to |lse| 2^-24, and every p of the row with it.  With its low word d, p = e^(u - d), u = l - lse, and
// p (c0 + c1 (u - d)) = e^u (c0' + c1' u) with c1' = c1 e^-d, c0' = (c0 - c1 d) e^-d: the row's coefficients take it, an element costs nothing more.
// TWO: with the low word.  Compiled apart, because a row's threads repeat its coefficients (2048 x 131072 bf16: 171 us, 177 with a test of the pointer there).
struct GradIn {
  const int32_t* labels;
  const float *lse, *entropy, *dlogp, *dentropy, *lse_low;
};
template <typename T>
struct GradOut { T* p; int64_t sk, sr, sc; };

template <bool TWO>
struct GradRow {
  float lse, c0, c1, at_label;
  int32_t y;   // class that receives at_label, -1: none, -2: the whole row is zero
  __device__ inline GradRow() : lse(0.f), c0(0.f), c1(0.f), at_label(0.f), y(-2) {}
  __device__ inline GradRow(const GradIn& g, int64_t i, int32_t classes) {
    y = g.labels ? g.labels[i] : -1;
    lse = g.lse[i];
    const float a = g.dlogp ? g.dlogp[i] : 0.f;
    const float b = g.dentropy ? g.dentropy[i] : 0.f;
    c0 = -a - (g.dentropy ? b * g.entropy[i] : 0.f);
    c1 = -b;
    at_label = a;
    if constexpr (TWO) {
      const float d = g.lse_low[i], f = expf(-d);
      c0 = f * fmaf(-c1, d, c0);
      c1 *= f;
    }
    if ((g.labels && y < 0) || lse == -INFINITY) y = -2;
    if (y >= classes) c0 = NAN;  // the whole row
  }
  __device__ inline float operator()(float l, int32_t c) const {
    const float u = max_nan(l - lse, -200.f);  // e^-200 is 0 in 32 bits, and (-inf) * 0 never arises
    const float p = ex2(u * kLog2e);
    float d = p * fmaf(c1, u, c0);
    if (c == y) d += at_label;
    return y == -2 ? 0.f : d;
  }
};

template <typename T> __device__ inline uint4 vec_pack(const float (&f)[16 / sizeof(T)]) {
  uint4 q;
  T* t = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int j = 0; j < (int)(16 / sizeof(T)); ++j) t[j] = from_float<T>(f[j]);
  return q;
}

// Rows of classes.  NT = 256: a block takes a chunk of a row, 32: a warp does (eight rows per block).  VECTORS: input and output rows have the
// same 16-byte phase (the host checks the strides), so that both move as vectors; UNIT: contiguous, consecutive lanes move consecutive elements; ANY: any stride.
enum : int { GRAD_VECTORS = 0, GRAD_UNIT = 1, GRAD_ANY = 2 };
template <typename T> __host__ __device__ constexpr int64_t grad_chunk(int mode, int NT) { return mode == GRAD_VECTORS ? (int64_t)NT * 4 * vec_n<T>() : (int64_t)NT * 8; }
template <typename T, int NT, int MODE, bool TWO>
__global__ void __launch_bounds__(256)
grad_row_kernel(LogitView<T> v, GradIn g, GradOut<T> out, FastDiv by_chunks, uint32_t units) {
  constexpr int N = vec_n<T>();
  const uint32_t unit = NT == 32 ? blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  if (unit >= units) return;
  const int t = threadIdx.x % NT;
  uint32_t chunk, r;
  const uint32_t i = by_chunks.div(unit, chunk), k = v.by_rows.div(i, r);
  const T* src = v.p + k * v.sk + r * v.sr;
  T* dst = out.p + k * out.sk + r * out.sr;
  if (MODE == GRAD_VECTORS) {
    const RowParts<T> rp(src, 1, v.classes);
    const int32_t q0 = (int32_t)chunk * NT * 4 + t;
    const uint4* from = reinterpret_cast<const uint4*>(src + rp.head) + q0;
    uint4* to = reinterpret_cast<uint4*>(dst + rp.head) + q0;
    uint4 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (q0 + e * NT < rp.nvec) x[e] = from[e * NT];
    const GradRow<TWO> row(g, i, v.classes);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (q0 + e * NT >= rp.nvec) break;
      float l[N];
      vec_unpack<T>(x[e], l);
      const int32_t c = rp.head + (q0 + e * NT) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) l[j] = row(l[j], c + j);
      to[e * NT] = vec_pack<T>(l);
    }
    if (chunk == 0) {  // both are shorter than a vector
      if (t < rp.head) dst[t] = from_float<T>(row(to_float(src[t]), t));
      const int64_t c = (int64_t)rp.tail0 + t;
      if (c < v.classes) dst[c] = from_float<T>(row(to_float(src[c]), (int32_t)c));
    }
  } else {
    const int64_t si = MODE == GRAD_UNIT ? 1 : v.sc, so = MODE == GRAD_UNIT ? 1 : out.sc;
    const int64_t c0 = (int64_t)chunk * 8 * NT + t;
    const int n = c0 < v.classes ? (int)min((int64_t)8, (v.classes - c0 + NT - 1) / NT) : 0;
    const T* from = src + c0 * si;
    T* to = dst + c0 * so;
    T x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) x[e] = from[e * NT * si];
    const GradRow<TWO> row(g, i, v.classes);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) to[e * NT * so] = from_float<T>(row(to_float(x[e]), (int32_t)c0 + e * NT));
  }
}

// Logits and gradient with the sample index contiguous: a thread owns R consecutive rows (a 16-byte vector, or one row where the strides do
// not allow it) and 8 classes of a block's 64.  block (32, 8), grid K * row blocks * class blocks.
template <typename T, int R, bool TWO>
__global__ void __launch_bounds__(256, R == 8 ? 3 : R == 1 ? 5 : 4)
grad_feature_kernel(LogitView<T> v, GradIn g, GradOut<T> out, uint32_t row_blocks, uint32_t class_blocks) {
  const uint32_t cb = blockIdx.x % class_blocks, kr = blockIdx.x / class_blocks, rb = kr % row_blocks, k = kr / row_blocks;
  const int64_t r0 = ((int64_t)rb * 32 + threadIdx.x) * R;
  if (r0 >= v.rows) return;
  const T* src = v.p + k * v.sk + r0;
  T* dst = out.p + k * out.sk + r0;
  GradRow<TWO> row[R];
#pragma unroll
  for (int j = 0; j < R; ++j)
    if (r0 + j < v.rows) row[j] = GradRow<TWO>(g, (int64_t)k * v.rows + r0 + j, v.classes);
  const int64_t c0 = (int64_t)cb * 64 + threadIdx.y;
  if (R > 1 && r0 + R <= v.rows) {
    constexpr int N = vec_n<T>();
    static_assert(R == 1 || R == N, "one vector of rows");
    const int n = c0 < v.classes ? (int)min((int64_t)8, (v.classes - c0 + 7) / 8) : 0;
    const T* from = src + c0 * v.sc;
    T* to = dst + c0 * out.sc;
    const int64_t si = 8 * v.sc, so = 8 * out.sc;
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // four vectors in flight at a time
      uint4 x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * h + e < n) x[e] = *reinterpret_cast<const uint4*>(from + (4 * h + e) * si);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * h + e < n) {
          const int32_t c = (int32_t)c0 + 8 * (4 * h + e);
          float l[N];
          vec_unpack<T>(x[e], l);
#pragma unroll
          for (int j = 0; j < N; ++j) l[j] = row[R > 1 ? j : 0](l[j], c);
          *reinterpret_cast<uint4*>(to + (4 * h + e) * so) = vec_pack<T>(l);
        }
    }
  } else {
    if constexpr (R == 1) {  // all loads in flight before the first store
      T x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c0 + 8 * e < v.classes) x[e] = src[(c0 + 8 * e) * v.sc];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c0 + 8 * e < v.classes) dst[(c0 + 8 * e) * out.sc] = from_float<T>(row[0](to_float(x[e]), (int32_t)c0 + 8 * e));
    } else {  // the last rows
      for (int e = 0; e < 8; ++e) {
        const int64_t c = c0 + 8 * e;
        if (c >= v.classes) break;
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (r0 + j < v.rows) dst[c * out.sc + j] = from_float<T>(row[j](to_float(src[c * v.sc + j]), (int32_t)c));
      }
    }
  }
}

}  // namespace lsam
