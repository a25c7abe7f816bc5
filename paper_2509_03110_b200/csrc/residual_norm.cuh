// residual_norm.cuh -- the end of one residual block and the start of the next in one pass: root-mean-square norm of the block's output, gate, residual
// scales, and the norm in front of the next block; and the gradient of all that.
//
//   c = b q, q = (mean b^2 + eps)^-1/2;   p = c w_post;   y = alpha x + beta act(z) p;   u = y r w_pre, r = (mean y^2 + eps)^-1/2
// Gradient, from dy and du (h = y r, dh = du w_pre):
//   g = dy + r (dh - h m1), m1 = mean(dh h);   dx = alpha g;   dz = beta g p act'(z);   dc = beta g act(z) w_post;   db = q (dc - c m2), m2 = mean(dc c)
//   dw_pre = sum over rows of du h;   dw_post = sum over rows of beta g act(z) c
// The floor is the bytes of the [rows, n] tensors: 32 x 256 x 4096 bf16 with a gate that is a tensor, 336 MB in 65 us forward (5.1 TB/s), 540 MB in 118 us
// back (4.6 TB/s, one block of 16 warps an SM, half of the issue slots).  The same rows in other forms: forward out = x + branch and its norm 48 us
// (5.6 TB/s), the norm alone 29 (4.6); back 128 and 97 us (3.1 and 2.1 TB/s), bound by the instructions of a row, in the form that tests for what is there.  Forward rows that do not fit
// registers (fp32 past 8192 columns) run at 1.2 to 3.1 TB/s: single elements, the inputs read again for every reduction.
// m2 depends on m1 through g, but linearly, so both come from three sums over a row that need
// no order among themselves:  S1 = sum dh h,  S2 = sum a (dy + r dh),  S3 = sum a r h  with a = beta act(z) w_post c:  m1 = S1 / n, m2 = (S2 - m1 S3) / n.
// (What cancels there is of the size of dc itself, whose own rounding is as large.)  The forward pass keeps two reductions: its sum of y^2 written that way
// would lose all digits of r where x and the branch cancel.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "tc_ptx.cuh"
#include "vec.cuh"

namespace lsam {

enum : int { GATE_NONE = 0, GATE_COLUMN = 1, GATE_ROW = 2, GATE_FULL = 3 };
enum : int { ACT_LINEAR = 0, ACT_SIGMOID = 1, ACT_TANH = 2 };

template <typename T>
struct RowsOf {  // [K, rows, n], columns contiguous
  T* p;
  int64_t sk;
  uint32_t sr;  // below 2^31: a row's place is one wide multiply-add behind its worker's
  __device__ inline T* worker(uint32_t k) const { return p + k * sk; }
  __device__ inline T* at(uint32_t k, uint32_t r) const { return worker(k) + (uint64_t)r * sr; }
};

template <typename T>
struct NormArgs {
  RowsOf<const T> x, branch, gate;  // gate: GATE_FULL only
  RowsOf<T> out, normed;
  const float *gate_f, *post_w, *pre_w;      // gate_f: GATE_COLUMN [K, n] or GATE_ROW [K, rows]
  int64_t gate_k, post_k, pre_k;             // their strides of a worker (0: shared)
  float *rstd_post, *rstd_pre;               // [K, rows], nullable
  int64_t rows, n;
  FastDiv by_rows;
  uint32_t total;  // K * rows
  int post, pre, kind, act;
  float alpha, beta, eps, inv_n;
};

// The sigmoid's exponential and reciprocal come from the special-function unit: off by a factor of 1 +- (2^-22 + 3 |z| 2^-24) at most.
__device__ inline float sigmoid_fast(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
__device__ inline float act_value(float z, int act) {
  if (act == ACT_SIGMOID) return sigmoid_fast(z);
  if (act == ACT_TANH) return tanhf(z);
  return z;
}
template <int E>
__device__ __forceinline__ void act_values(float (&v)[E], int act) {
  if (act == ACT_SIGMOID) {
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = sigmoid_fast(v[j]);
  } else if (act == ACT_TANH) {
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = tanhf(v[j]);
  }
}
// The slope from the value, as c0 + v (c1 - c2 v): 1, v (1 - v) or 1 - v^2.
struct Slope {
  float c0, c1, c2;
  __device__ explicit Slope(int act) : c0(act == ACT_SIGMOID ? 0.f : 1.f), c1(act == ACT_SIGMOID ? 1.f : 0.f), c2(act == ACT_LINEAR ? 0.f : 1.f) {}
  __device__ inline float operator()(float v) const { return fmaf(v, fmaf(-c2, v, c1), c0); }
};

// Columns of a thread: E of them, as 16-byte vectors NT vectors apart (n is then a multiple of a vector), or one by one NT apart.  `p` of the calls is the
// row's start.
template <typename T, int NT, int E, bool VEC>
struct NormCols {
  static constexpr int N = VEC ? vec_n<T>() : 1, Q = E / N;
  int off, left;  // the thread's first column, and how many there are from it on
  struct Raw {  // as stored
    typename std::conditional<VEC, uint4, T>::type q[Q];
  };
  __device__ NormCols(int t, int64_t n) : off(t * N), left((int)n - t * N) {}
  static __device__ constexpr int place(int j) { return j / N * NT * N + j % N; }  // of column j behind the first
  __device__ inline bool have(int j) const { return place(j) < left; }
  __device__ inline int col(int j) const { return off + place(j); }
  __device__ inline void fetch(const T* p, Raw& r) const {
    p += off;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = q * NT * N;
      if constexpr (VEC) r.q[q] = c < left ? *reinterpret_cast<const uint4*>(p + c) : make_uint4(0u, 0u, 0u, 0u);
      else r.q[q] = c < left ? p[c] : from_float<T>(0.f);
    }
  }
  // the thread's vectors, asynchronously, `apart` 16-byte words apart in shared memory
  __device__ inline void copy(const T* p, uint4* to, int apart) const {
    p += off;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = q * NT * N;
      const uint32_t bytes = c < left ? 16u : 0u;  // zeros behind the row
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to + q * apart)), "l"(c < left ? p + c : p - off), "r"(bytes) : "memory");
    }
  }
  __device__ inline void unpack(const Raw& r, float (&v)[E]) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if constexpr (VEC) {
        float f[N];
        vec_unpack<T>(r.q[q], f);
#pragma unroll
        for (int j = 0; j < N; ++j) v[q * N + j] = f[j];
      } else {
        v[q] = to_float(r.q[q]);
      }
    }
  }
  __device__ inline void unpack(const Raw& r, uint64_t (&v)[E / 2]) const {
    float f[E];
    unpack(r, f);
    pairs(f, v);
  }
  static __device__ inline void pairs(const float (&f)[E], uint64_t (&v)[E / 2]) {
#pragma unroll
    for (int j = 0; j < E / 2; ++j) v[j] = pack2(f[2 * j], f[2 * j + 1]);
  }
  __device__ inline void load(const T* p, float (&v)[E]) const {
    Raw r;
    fetch(p, r);
    unpack(r, v);
  }
  __device__ inline void store(T* p, const float (&v)[E]) const {
    p += off;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = q * NT * N;
      if (c >= left) continue;
      if constexpr (VEC) {
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = v[q * N + j];
        *reinterpret_cast<uint4*>(p + c) = vec_pack<T>(f);
      } else {
        p[c] = from_float<T>(v[q]);
      }
    }
  }
  __device__ inline void store(T* p, const uint64_t (&v)[E / 2]) const {
    float f[E];
#pragma unroll
    for (int j = 0; j < E / 2; ++j) unpack2(v[j], f[2 * j], f[2 * j + 1]);
    store(p, f);
  }
  __device__ inline void load_pairs(const float* p, uint64_t (&v)[E / 2], float other) const {
    float f[E];
    load_f(p, f, other);
    pairs(f, v);
  }
  // a vector of fp32 parameters, or `other` where there is none
  __device__ inline void load_f(const float* p, float (&v)[E], float other) const {
    p = p ? p + off : p;
    if (VEC && p && !(reinterpret_cast<uintptr_t>(p) & 15)) {
#pragma unroll
      for (int q = 0; q < E; q += 4) {
        const int c = place(q);
        const float4 f = c < left ? __ldg(reinterpret_cast<const float4*>(p + c)) : make_float4(other, other, other, other);
        v[q] = f.x; v[q + 1] = f.y; v[q + 2] = f.z; v[q + 3] = f.w;
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = p && have(j) ? __ldg(p + place(j)) : other;
  }
};

// Sum over the NT threads of a row, in every one of them.  One barrier: consecutive sums go to different arrays, so that the next one's barrier stands between
// the reads of this one and the next writes to its array.
template <int NT>
__device__ inline float group_sum(float v, float* smem) {
  v = warp_sum(v);
  if constexpr (NT > 32) {
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 32; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(smem + i);
      v += (f.x + f.y) + (f.z + f.w);
    }
  }
  return v;
}

// A row per NT threads, the row in registers between its two reductions: every tensor is read or written once.  Blocks walk the rows, the next one on its way into
// shared memory (every thread its own vectors, so no barrier) while this one is worked on: 64 registers, and four rows of 4096 16-bit columns on an SM with
// four more coming.  FORM_FULL: both norms and a gate that is a tensor, without a test of what is there.
constexpr int norm_threads(int NT) { return NT == 32 ? 128 : NT; }
enum : int { FORM_ANY = 0, FORM_FULL = 1, FORM_COLUMN = 2 };
template <typename T, int E, bool VEC> constexpr int norm_ring(int NT) { return VEC ? 2 * 3 * (E / vec_n<T>()) * norm_threads(NT) * 16 : 0; }
template <typename T, int NT, int E, bool VEC, int FORM>
__global__ void __launch_bounds__(norm_threads(NT), E <= 2 * vec_n<T>() ? 1024 / norm_threads(NT) : 1)
residual_norm_kernel(NormArgs<T> a) {
  constexpr int THREADS = NT == 32 ? 128 : NT, ROWS = THREADS / NT, P = E / 2;
  extern __shared__ uint4 norm_ring_words[];  // [2][branch, x, gate][vectors][threads]
  __shared__ __align__(16) float smem[2][2][NT > 32 ? NT / 32 : 4];  // a row's two sums, those of the next row apart
  using Cols = NormCols<T, NT, E, VEC>;
  const Cols w((int)(threadIdx.x % NT), a.n);
  const bool has_b = FORM == FORM_FULL || a.branch.p, full = FORM == FORM_FULL || a.kind == GATE_FULL, post = FORM == FORM_FULL || a.post, pre = FORM == FORM_FULL || a.pre;
  const uint32_t step = gridDim.x * ROWS;
  const auto fetch = [&](uint32_t i, int stage) {
    if constexpr (VEC) {
      if (i < a.total) {
        uint32_t r;
        const uint32_t k = a.by_rows.div(i, r);
        uint4* to = norm_ring_words + stage * (3 * Cols::Q * THREADS) + threadIdx.x;
        if (has_b) w.copy(a.branch.at(k, r), to, THREADS);
        w.copy(a.x.at(k, r), to + Cols::Q * THREADS, THREADS);
        if (full) w.copy(a.gate.at(k, r), to + 2 * Cols::Q * THREADS, THREADS);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  };
  uint32_t i = NT == 32 ? blockIdx.x * ROWS + (threadIdx.x >> 5) : blockIdx.x;
  fetch(i, 0);
  for (int stage = 0; i < a.total; i += step, stage ^= 1) {
    uint32_t r;
    const uint32_t k = a.by_rows.div(i, r);
    const uint4* from = norm_ring_words + stage * (3 * Cols::Q * THREADS) + threadIdx.x;
    fetch(i + step, stage ^ 1);
    if (VEC) asm volatile("cp.async.wait_group 1;" ::: "memory");
    const auto take = [&](const RowsOf<const T>& t, int slot, uint64_t (&v)[P]) {
      typename Cols::Raw raw;
      if constexpr (VEC) {
#pragma unroll
        for (int q = 0; q < Cols::Q; ++q) raw.q[q] = from[(slot * Cols::Q + q) * THREADS];
      } else {
        w.fetch(t.at(k, r), raw);
      }
      w.unpack(raw, v);
    };
    uint64_t y[P], v[P];
    if (has_b) {
      take(a.branch, 0, y);
      float f = a.beta;
      if (FORM != FORM_FULL && a.kind == GATE_ROW) f *= act_value(__ldg(a.gate_f + i), a.act);
      if (post) {
        uint64_t s = 0;
#pragma unroll
        for (int j = 0; j < P; ++j) s = fma2(y[j], y[j], s);
        float s0, s1;
        unpack2(s, s0, s1);
        const float q = 1.f / sqrtf(group_sum<NT>(s0 + s1, smem[stage][0]) * a.inv_n + a.eps);
        if (w.off == 0 && a.rstd_post) a.rstd_post[i] = q;
        w.load_pairs(a.post_w ? a.post_w + k * a.post_k : nullptr, v, 1.f);
        f *= q;
#pragma unroll
        for (int j = 0; j < P; ++j) y[j] = mul2(y[j], v[j]);
      }
      if (full || (FORM != FORM_FULL && a.kind == GATE_COLUMN)) {
        if (full) take(a.gate, 2, v);
        else w.load_pairs(a.gate_f + k * a.gate_k, v, 0.f);
        float z[E];
#pragma unroll
        for (int j = 0; j < P; ++j) unpack2(v[j], z[2 * j], z[2 * j + 1]);
        act_values(z, a.act);
        Cols::pairs(z, v);
#pragma unroll
        for (int j = 0; j < P; ++j) y[j] = mul2(y[j], v[j]);
      }
      take(a.x, 1, v);
      const uint64_t f2 = pack2(f, f), alpha2 = pack2(a.alpha, a.alpha);
#pragma unroll
      for (int j = 0; j < P; ++j) y[j] = fma2(alpha2, v[j], mul2(f2, y[j]));
      w.store(a.out.at(k, r), y);
    } else {
      take(a.x, 1, y);
    }
    if (pre) {
      uint64_t s = 0;
      if (w.have(E - 1)) {
#pragma unroll
        for (int j = 0; j < P; ++j) s = fma2(y[j], y[j], s);
      } else {  // an infinite gate times the zeros behind the row is no part of it
#pragma unroll
        for (int j = 0; j < P; ++j) {
          float y0, y1;
          unpack2(y[j], y0, y1);
          const uint64_t m = pack2(w.have(2 * j) ? y0 : 0.f, w.have(2 * j + 1) ? y1 : 0.f);
          s = fma2(m, m, s);
        }
      }
      float s0, s1;
      unpack2(s, s0, s1);
      const float q = 1.f / sqrtf(group_sum<NT>(s0 + s1, smem[stage][1]) * a.inv_n + a.eps);
      if (w.off == 0 && a.rstd_pre) a.rstd_pre[i] = q;
      w.load_pairs(a.pre_w ? a.pre_w + k * a.pre_k : nullptr, v, 1.f);
      const uint64_t q2 = pack2(q, q);
#pragma unroll
      for (int j = 0; j < P; ++j) y[j] = mul2(mul2(y[j], q2), v[j]);
      w.store(a.normed.at(k, r), y);
    }
  }
}

// Rows that do not fit into registers: the inputs are read again for every reduction (out may be x, so nothing is stored before the last one).
template <typename T>
__global__ void __launch_bounds__(1024)
residual_norm_long_kernel(NormArgs<T> a) {
  __shared__ __align__(16) float smem[2][32];
  const uint32_t i = blockIdx.x;
  uint32_t r;
  const uint32_t k = a.by_rows.div(i, r);
  const T *x = a.x.at(k, r), *b = a.branch.p ? a.branch.at(k, r) : nullptr, *z = a.kind == GATE_FULL ? a.gate.at(k, r) : nullptr;
  const float* zc = a.kind == GATE_COLUMN ? a.gate_f + k * a.gate_k : nullptr;
  const float *pw = a.post_w ? a.post_w + k * a.post_k : nullptr, *nw = a.pre_w ? a.pre_w + k * a.pre_k : nullptr;
  float f = a.beta, q = 1.f;
  if (a.kind == GATE_ROW) f *= act_value(__ldg(a.gate_f + i), a.act);
  if (b && a.post) {
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < a.n; c += 1024) { const float v = to_float(b[c]); s = fmaf(v, v, s); }
    q = 1.f / sqrtf(group_sum<1024>(s, smem[0]) * a.inv_n + a.eps);
    if (threadIdx.x == 0 && a.rstd_post) a.rstd_post[i] = q;
  }
  const auto value = [&](int64_t c) {
    const float v = to_float(x[c]);
    if (!b) return v;
    float g = f;
    if (z) g *= act_value(to_float(z[c]), a.act);
    if (zc) g *= act_value(__ldg(zc + c), a.act);
    return fmaf(a.alpha, v, g * (a.post ? to_float(b[c]) * q * (pw ? __ldg(pw + c) : 1.f) : to_float(b[c])));
  };
  float n = 0.f;
  if (a.pre) {
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < a.n; c += 1024) { const float v = value(c); s = fmaf(v, v, s); }
    n = 1.f / sqrtf(group_sum<1024>(s, smem[1]) * a.inv_n + a.eps);
    if (threadIdx.x == 0 && a.rstd_pre) a.rstd_pre[i] = n;
  }
  T *out = b ? a.out.at(k, r) : nullptr, *normed = a.pre ? a.normed.at(k, r) : nullptr;
  for (int64_t c = threadIdx.x; c < a.n; c += 1024) {
    const float v = value(c);
    if (out) out[c] = from_float<T>(v);
    if (normed) normed[c] = from_float<T>(v * n * (nw ? __ldg(nw + c) : 1.f));
  }
}

// ------------------------------------------------------------------------------------------------ gradient
template <typename T>
struct NormGradArgs {
  RowsOf<const T> y, branch, gate, dy, du;  // dy, du: nullable
  RowsOf<T> dx, db, dz;                     // dz: GATE_FULL only
  const float *gate_f, *post_w, *pre_w, *rstd_post, *rstd_pre;
  int64_t gate_k, post_k, pre_k;
  float* dz_row;     // GATE_ROW [K, rows]
  float2* means;     // [K, rows]: m1, m2; null where neither is needed
  float* part;       // [slots, which, ld_part] column sums of a strip: dw_pre, dw_post, dz of GATE_COLUMN, those that are wanted
  int64_t rows, n, strip;  // strip: rows of one
  int64_t ld_part, per;    // per: columns of a block of a cluster
  FastDiv by_rows;
  uint32_t total;
  int32_t strips, which;
  int want_pre, want_post, want_gate;  // 1 + place in `part`, or 0
  int post, pre, kind, act;
  float alpha, beta, inv_n;
};

constexpr int kGradRanks = 8;  // blocks of a cluster, at most

// The whole gradient in one pass.  A block walks a strip of the K * rows rows, the next row's vectors of every tensor in flight while this one is worked on; a row
// lies in the registers of NT threads (8 columns each) across its one reduction, and the column sums stay there until the strip, or a worker's part of
// it, ends.  Strips are equal shares of all rows, whichever worker they belong to; the sums of block b for worker k go to slot b + k (b and k never fall
// together, so no slot is used twice).  NT = 32: four warps a block, which take turns and are added at the end.
// FORM_FULL and FORM_COLUMN: both norms, dout, and every tensor's gradient wanted, with a gate that is a tensor, or one for every column or none: without
// a test of what is there.
// TURNS: rows that a block works on at a time.  Rows of more than 4096 columns are shared by a cluster of blocks, `per` columns each (CLUSTER), which send
// their sums to one another.
// STARVED (self-test): the sums of the last block never reach the first one in the third row of every strip, and waits are short.
template <typename T, int NT, bool VEC, bool CLUSTER, int FORM, bool STARVED = false>
__global__ void __launch_bounds__(norm_threads(NT), 512 / norm_threads(NT))
residual_norm_grad_fused_kernel(NormGradArgs<T> a) {
  constexpr int E = 8, P = E / 2, TURNS = NT == 32 ? 4 : 1, WARPS = NT / 32, RANKS = CLUSTER ? kGradRanks : 1;
  __shared__ __align__(16) float sums[2][RANKS][3][WARPS < 4 ? 4 : WARPS];
  __shared__ float join[TURNS > 1 ? TURNS : 1][TURNS > 1 ? 32 : 1];
  grid_dep_sync();
  using Cols = NormCols<T, NT, E, VEC>;
  uint32_t rank = 0, ranks = 1;
  if (CLUSTER) {
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    // columns of this block; from here on every pointer starts there
    const int64_t c0 = (int64_t)rank * a.per;
    a.n = min(a.per, a.n - c0);
    a.y.p += c0; a.du.p += c0; a.dy.p = a.dy.p ? a.dy.p + c0 : nullptr; a.branch.p = a.branch.p ? a.branch.p + c0 : nullptr; a.gate.p += c0;
    a.dx.p = a.dx.p ? a.dx.p + c0 : nullptr; a.db.p = a.db.p ? a.db.p + c0 : nullptr; a.dz.p = a.dz.p ? a.dz.p + c0 : nullptr;
    a.post_w = a.post_w ? a.post_w + c0 : nullptr; a.pre_w = a.pre_w ? a.pre_w + c0 : nullptr;
    if (a.kind == GATE_COLUMN) a.gate_f += c0;
    a.part += c0;
  }
  // Sums travel as asynchronous stores that count on the receiver's barrier: a barrier of the cluster, whose release waits for every global store before it, took
  // 1.5 us a row.  Nobody can send for the row after next before every warp has sent for the next one, so two sets of sums are enough.  The wait is
  // bounded.  A thread whose wait runs out goes on with NaN and neither sends nor waits again: whatever it sent would land, too early, in a set that another
  // block may still read.  So the others' next row stays incomplete, their waits run out in turn, and no row is made of a mixture.
  __shared__ uint64_t arrived[2];
  __shared__ volatile int never;
  uint32_t phase = 0;
  int dead = 0;
  if constexpr (CLUSTER) {
    if (threadIdx.x == 0) {
      tc::mbar_init(&arrived[0], 1);
      tc::mbar_init(&arrived[1], 1);
      never = 0;
      tc::fence_barrier_init();
    }
    tc::cluster_sync_all();
  }
  const uint32_t block = blockIdx.x / ranks;
  const Cols w((int)(threadIdx.x % NT), a.n);
  const int turn = TURNS > 1 ? threadIdx.x >> 5 : 0;
  const int64_t first = (int64_t)block * a.strip, end = min((int64_t)a.total, first + a.strip);
  constexpr bool ALL = FORM != FORM_ANY;
  const bool full = FORM == FORM_FULL || (!ALL && a.kind == GATE_FULL), has_b = ALL || a.branch.p, has_dy = ALL || a.dy.p, pre = ALL || a.pre, post = ALL || a.post;
  const bool row_gate = !ALL && a.kind == GATE_ROW, column_gate = FORM == FORM_COLUMN ? a.kind == GATE_COLUMN : !ALL && a.kind == GATE_COLUMN;
  const Slope slope(a.act);
  typename Cols::Raw ry, ru, rg, rb, rz;
  float rp_next = 0.f, q_next = 1.f, v_next = 1.f;
  const auto fetch = [&](uint32_t k, uint32_t r, uint32_t i) {
    if (pre) { w.fetch(a.y.at(k, r), ry); w.fetch(a.du.at(k, r), ru); rp_next = __ldg(a.rstd_pre + i); }
    if (has_dy) w.fetch(a.dy.at(k, r), rg);
    if (has_b) w.fetch(a.branch.at(k, r), rb);
    if (full) w.fetch(a.gate.at(k, r), rz);
    if (post) q_next = __ldg(a.rstd_post + i);
    if (row_gate) v_next = __ldg(a.gate_f + i);
  };
  uint32_t r0;
  uint32_t k = a.by_rows.div((uint32_t)first, r0);
  int64_t base = first - r0;  // row 0 of worker k
  int parity = 0;
  for (int64_t lo = first; lo < end;) {
    const int64_t hi = min(end, base + a.rows);  // this worker's part
    uint64_t pw[P], nw[P], v[P], acc[3][P];
    {
      float f[E];
      w.load_f(a.post_w ? a.post_w + k * a.post_k : nullptr, f, 1.f);
      Cols::pairs(f, pw);
      w.load_f(a.pre_w ? a.pre_w + k * a.pre_k : nullptr, f, 1.f);
      Cols::pairs(f, nw);
      w.load_f(column_gate ? a.gate_f + k * a.gate_k : nullptr, f, 1.f);
      if (column_gate) act_values(f, a.act);
      Cols::pairs(f, v);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) acc[0][j] = acc[1][j] = acc[2][j] = 0;
    // the rows of a part are dealt to the turns by their place in the strip
    const int64_t i0 = first + turn + (lo - first + TURNS - 1 - turn) / TURNS * TURNS;
    if (i0 < hi) fetch(k, (uint32_t)(i0 - base), (uint32_t)i0);
    for (int64_t i = i0; i < hi; i += TURNS) {
      const uint32_t r = (uint32_t)(i - base);
      uint64_t h[P], g[P], c[P];
      const float rp = rp_next, q = q_next;
      const uint64_t rp2 = pack2(rp, rp), q2 = pack2(q, q);
      uint64_t s1 = 0, s2 = 0, s3 = 0;
      if (has_dy) w.unpack(rg, g);
      else
#pragma unroll
        for (int j = 0; j < P; ++j) g[j] = 0;
      if (pre) {
        uint64_t u[P];
        w.unpack(ry, h);
        w.unpack(ru, u);
#pragma unroll
        for (int j = 0; j < P; ++j) {
          h[j] = mul2(h[j], rp2);
          acc[0][j] = fma2(u[j], h[j], acc[0][j]);
          const uint64_t dh = mul2(u[j], nw[j]);
          s1 = fma2(dh, h[j], s1);
          g[j] = fma2(rp2, dh, g[j]);
          h[j] = mul2(h[j], rp2);
        }
      } else {
#pragma unroll
        for (int j = 0; j < P; ++j) h[j] = 0;
      }
      float gate = 1.f;
      if (has_b) {
        w.unpack(rb, c);
        if (full) {
          float z[E];
          w.unpack(rz, z);
          act_values(z, a.act);
          Cols::pairs(z, v);
        }
        if (row_gate) gate = act_value(v_next, a.act);
#pragma unroll
        for (int j = 0; j < P; ++j) {
          c[j] = mul2(c[j], q2);
          const uint64_t p = mul2(mul2(c[j], pw[j]), v[j]);
          s2 = fma2(p, g[j], s2);
          s3 = fma2(p, h[j], s3);
        }
      }
      if (i + TURNS < hi) fetch(k, r + TURNS, (uint32_t)(i + TURNS));
      float t[3];
      {
        float x, y;
        unpack2(s1, x, y); t[0] = x + y;
        unpack2(s2, x, y); t[1] = x + y;
        unpack2(s3, x, y); t[2] = x + y;
      }
      if constexpr (WARPS > 1) {
        // four sums (the last one nothing) by halves: lanes 0, 8, 16, 24 end with one each
        const int lane = threadIdx.x & 31;
        float x = ((lane & 16) ? t[2] : t[0]) + __shfl_xor_sync(~0u, (lane & 16) ? t[0] : t[2], 16);
        float y = ((lane & 16) ? 0.f : t[1]) + __shfl_xor_sync(~0u, (lane & 16) ? t[1] : 0.f, 16);
        x = ((lane & 8) ? y : x) + __shfl_xor_sync(~0u, (lane & 8) ? x : y, 8);
        x += __shfl_xor_sync(~0u, x, 4);
        x += __shfl_xor_sync(~0u, x, 2);
        x += __shfl_xor_sync(~0u, x, 1);
        if ((lane & 7) == 0 && lane < 24 && !dead) {
          float* to = &sums[parity][CLUSTER ? rank : 0][lane >> 3][threadIdx.x >> 5];
          if constexpr (CLUSTER) {
            const uint32_t at = tc::smem_u32(to), bar = tc::smem_u32(&arrived[parity]);
            for (uint32_t c = STARVED && rank == ranks - 1 && i == first + 2 ? 1u : 0u; c < ranks; ++c)
              asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(tc::map_to_cta(at, c)), "f"(x), "r"(tc::map_to_cta(bar, c)) : "memory");
          } else {
            *to = x;
          }
        }
        // the other half was read before it
        if constexpr (CLUSTER) {
          if (!dead) {
            if (threadIdx.x == 0) tc::mbar_expect_tx(&arrived[parity], ranks * WARPS * 12);
            if (!tc::mbar_wait_limit(&arrived[parity], phase, &never, STARVED ? 1u << 13 : tc::kSpinLimit)) dead = 1;
          }
          if (parity) phase ^= 1u;
        } else {
          __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) t[e] = 0.f;
        for (uint32_t c = 0; c < ranks; ++c)
#pragma unroll
          for (int e = 0; e < 3; ++e)
#pragma unroll
            for (int x = 0; x < WARPS; x += 4) {
              const float4 f = *reinterpret_cast<const float4*>(&sums[parity][CLUSTER ? c : 0][e][x]);
              t[e] += (f.x + f.y) + (f.z + f.w);
            }
        if (CLUSTER && dead) t[0] = t[1] = t[2] = NAN;
        parity ^= 1;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) t[e] = warp_sum(t[e]);
      }
      // a gate per row stays out of the sums (v is 1): its own gradient is made of them
      const float m1 = t[0] * a.inv_n, gp = t[1] - m1 * t[2], m2 = a.beta * gate * gp * a.inv_n;
      if (row_gate && a.dz_row && w.off == 0 && rank == 0) a.dz_row[i] = a.beta * slope(gate) * gp;
      const uint64_t n1 = pack2(-m1, -m1), n2 = pack2(-m2, -m2), bg = pack2(a.beta * gate, a.beta * gate), alpha2 = pack2(a.alpha, a.alpha);
      const uint64_t c0 = pack2(slope.c0, slope.c0), c1 = pack2(slope.c1, slope.c1), c2 = pack2(-slope.c2, -slope.c2);
#pragma unroll
      for (int j = 0; j < P; ++j) g[j] = fma2(h[j], n1, g[j]);
      if (has_b) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const uint64_t e = mul2(bg, g[j]), d = mul2(e, v[j]), ew = mul2(e, pw[j]);
          h[j] = mul2(mul2(ew, c[j]), fma2(v[j], fma2(c2, v[j], c1), c0));  // dz
          acc[1][j] = fma2(d, c[j], acc[1][j]);
          if (FORM != FORM_FULL) acc[2][j] = add2(acc[2][j], h[j]);
          c[j] = post ? mul2(q2, fma2(c[j], n2, mul2(ew, v[j]))) : d;
          g[j] = mul2(g[j], alpha2);
        }
        if (ALL || a.db.p) w.store(a.db.at(k, r), c);
        if (full && (ALL || a.dz.p)) w.store(a.dz.at(k, r), h);
      }
      if (ALL || a.dx.p) w.store(a.dx.at(k, r), g);
    }
    const int want[3] = {a.want_pre, a.want_post, a.want_gate};
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      if (!want[s]) continue;
      float* to = a.part + (((int64_t)block + k) * a.which + want[s] - 1) * a.ld_part;
      float f[E];
#pragma unroll
      for (int j = 0; j < P; ++j) unpack2(acc[s][j], f[2 * j], f[2 * j + 1]);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        if constexpr (TURNS > 1) {
          const int lane = threadIdx.x & 31;
          __syncthreads();
          join[turn][lane] = f[j];
          __syncthreads();
          if (turn == 0 && w.have(j)) to[w.col(j)] = ((join[0][lane] + join[1][lane]) + join[2][lane]) + join[3][lane];
        } else {
          if (w.have(j)) to[w.col(j)] = f[j];
        }
      }
    }
    lo = hi;
    base += a.rows;
    ++k;
  }
  // no block leaves while another's sums may still be on their way to it: all have sent what they will, and what a block has not waited for gets a millisecond to land
  if constexpr (CLUSTER) {
    tc::cluster_sync_all();
    if (dead) {
      const long long t0 = clock64();
      while (clock64() - t0 < 2000000LL) { }
    }
  }
}

// Rows of more columns than a cluster holds: two passes.
// The two means of every row, and the gradient of a gate per row.  A block of 256 threads per row.
template <typename T>
__global__ void __launch_bounds__(256)
residual_norm_grad_rows_kernel(NormGradArgs<T> a) {
  __shared__ __align__(16) float smem[3][8];
  const uint32_t i = blockIdx.x;
  uint32_t r;
  const uint32_t k = a.by_rows.div(i, r);
  const T *y = a.pre ? a.y.at(k, r) : nullptr, *du = a.pre ? a.du.at(k, r) : nullptr, *dy = a.dy.p ? a.dy.at(k, r) : nullptr;
  const T *b = a.branch.p ? a.branch.at(k, r) : nullptr, *z = a.kind == GATE_FULL ? a.gate.at(k, r) : nullptr;
  const float* zc = a.kind == GATE_COLUMN ? a.gate_f + k * a.gate_k : nullptr;
  const float *pw = a.post_w ? a.post_w + k * a.post_k : nullptr, *nw = a.pre_w ? a.pre_w + k * a.pre_k : nullptr;
  const float rp = a.pre ? a.rstd_pre[i] : 0.f, q = a.post ? a.rstd_post[i] : 1.f;
  const bool branch = b && (a.post || a.kind == GATE_ROW);
  float s1 = 0.f, s2 = 0.f, s3 = 0.f;
  for (int64_t c = threadIdx.x; c < a.n; c += 256) {
    float h = 0.f, dh = 0.f;
    if (a.pre) {
      h = to_float(y[c]) * rp;
      dh = to_float(du[c]) * (nw ? __ldg(nw + c) : 1.f);
      s1 = fmaf(dh, h, s1);
    }
    if (branch) {
      float v = to_float(b[c]) * q * (pw ? __ldg(pw + c) : 1.f);
      if (z) v *= act_value(to_float(z[c]), a.act);
      if (zc) v *= act_value(__ldg(zc + c), a.act);
      s2 = fmaf(v, fmaf(rp, dh, dy ? to_float(dy[c]) : 0.f), s2);
      s3 = fmaf(v, rp * h, s3);
    }
  }
  const float m1 = a.pre ? group_sum<256>(s1, smem[0]) * a.inv_n : 0.f;
  float m2 = 0.f;
  if (branch) {
    const float gp = group_sum<256>(s2, smem[1]) - m1 * group_sum<256>(s3, smem[2]);  // sum of g p, or of g act(z) p
    float v = 1.f;
    if (a.kind == GATE_ROW) {
      v = act_value(__ldg(a.gate_f + i), a.act);
      if (threadIdx.x == 0 && a.dz_row) a.dz_row[i] = a.beta * Slope(a.act)(v) * gp;
    }
    m2 = a.beta * v * gp * a.inv_n;
  }
  if (threadIdx.x == 0) a.means[i] = make_float2(m1, m2);
}

// Columns of a strip of rows, with everything that a row has to say known: grid (column chunks, strips, workers).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
residual_norm_grad_kernel(NormGradArgs<T> a) {
  constexpr int E = VEC ? vec_n<T>() : 4;
  grid_dep_sync();
  const int64_t c0 = (int64_t)blockIdx.x * 256 * E;
  const NormCols<T, 256, E, VEC> w((int)threadIdx.x, a.n - c0);
  const uint32_t k = blockIdx.z;
  const int64_t r0 = (int64_t)blockIdx.y * a.strip, r1 = min(a.rows, r0 + a.strip);
  const Slope slope(a.act);
  float pw[E], nw[E], zc[E], acc[3][E];
  w.load_f(a.post_w ? a.post_w + k * a.post_k + c0 : nullptr, pw, 1.f);
  w.load_f(a.pre_w ? a.pre_w + k * a.pre_k + c0 : nullptr, nw, 1.f);
  w.load_f(a.kind == GATE_COLUMN ? a.gate_f + k * a.gate_k + c0 : nullptr, zc, 0.f);
#pragma unroll
  for (int j = 0; j < E; ++j) {
    zc[j] = act_value(zc[j], a.act);
    acc[0][j] = acc[1][j] = acc[2][j] = 0.f;
  }
  for (int64_t r = r0; r < r1; ++r) {
    const int64_t i = k * a.rows + r;
    const float2 m = a.means ? a.means[i] : make_float2(0.f, 0.f);
    const float rp = a.pre ? a.rstd_pre[i] : 0.f, q = a.post ? a.rstd_post[i] : 1.f;
    float g[E], t[E], y[E], b[E], z[E];
    if (a.dy.p) w.load(a.dy.at(k, r) + c0, g);
    else
#pragma unroll
      for (int j = 0; j < E; ++j) g[j] = 0.f;
    if (a.pre) { w.load(a.du.at(k, r) + c0, t); w.load(a.y.at(k, r) + c0, y); }
    if (a.branch.p) w.load(a.branch.at(k, r) + c0, b);
    if (a.kind == GATE_FULL) w.load(a.gate.at(k, r) + c0, z);
    if (a.pre) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float h = y[j] * rp;
        acc[0][j] = fmaf(t[j], h, acc[0][j]);
        g[j] = fmaf(rp, fmaf(-h, m.x, t[j] * nw[j]), g[j]);
      }
    }
    if (a.branch.p) {
      const float vr = a.kind == GATE_ROW ? act_value(__ldg(a.gate_f + i), a.act) : 1.f;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float v = a.kind == GATE_FULL ? act_value(z[j], a.act) : a.kind == GATE_COLUMN ? zc[j] : vr;
        const float c = b[j] * q, bg = a.beta * g[j], d = bg * v;
        const float dz = bg * c * pw[j] * slope(v);
        z[j] = dz;
        acc[1][j] = fmaf(d, c, acc[1][j]);
        acc[2][j] += dz;
        b[j] = a.post ? q * fmaf(-c, m.y, d * pw[j]) : d;
        g[j] *= a.alpha;
      }
      if (a.db.p) w.store(a.db.at(k, r) + c0, b);
      if (a.kind == GATE_FULL && a.dz.p) w.store(a.dz.at(k, r) + c0, z);
    }
    if (a.dx.p) w.store(a.dx.at(k, r) + c0, g);
  }
  const int want[3] = {a.want_pre, a.want_post, a.want_gate};
#pragma unroll
  for (int s = 0; s < 3; ++s)
    if (want[s]) {
      float* to = a.part + (((int64_t)k * a.strips + blockIdx.y) * a.which + want[s] - 1) * a.ld_part + c0;
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (w.have(j)) to[w.col(j)] = acc[s][j];
    }
}

// The strips' column sums, in their order: over a worker's slots, or over all workers' where the parameter is shared.
struct NormSumArgs {
  const float* part;
  float* to[3];
  int shared[3];
  int64_t n, rows, strip, ld_part;  // strip: rows of a block's share of all of them
  int32_t strips, which, K;  // strips: of a worker, 0 where strips are shares of all rows
};
constexpr int kNormSumLanes = 8;
__global__ void __launch_bounds__(32 * kNormSumLanes)
residual_norm_grad_sum_kernel(NormSumArgs a) {
  __shared__ float4 smem[kNormSumLanes][32];
  grid_dep_sync();
  const int64_t c = ((int64_t)blockIdx.x * 32 + threadIdx.x) * 4;
  const int s = blockIdx.y;
  const bool shared = s == 0 ? a.shared[0] : s == 1 ? a.shared[1] : a.shared[2];
  const int k0 = blockIdx.z, k1 = shared ? a.K : k0 + 1;
  if (shared ? k0 > 0 : k0 >= a.K) return;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < a.n && a.rows > 0)
    for (int k = k0; k < k1; ++k) {
      const int64_t first = a.strips ? (int64_t)k * a.strips : (int64_t)k * a.rows / a.strip + k;
      const int64_t last = a.strips ? first + a.strips - 1 : ((int64_t)(k + 1) * a.rows - 1) / a.strip + k;
      for (int64_t j = first + threadIdx.y; j <= last; j += kNormSumLanes) {
        const float4 f = *reinterpret_cast<const float4*>(a.part + (j * a.which + s) * a.ld_part + c);
        v.x += f.x; v.y += f.y; v.z += f.z; v.w += f.w;
      }
    }
  smem[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.y < 4 && c + threadIdx.y < a.n) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < kNormSumLanes; ++j) t += reinterpret_cast<const float*>(&smem[j][threadIdx.x])[threadIdx.y];
    float* to = s == 0 ? a.to[0] : s == 1 ? a.to[1] : a.to[2];
    to[(int64_t)k0 * a.n + c + threadIdx.y] = t;
  }
}

}  // namespace lsam
