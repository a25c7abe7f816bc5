// head_score.cuh -- scores of activations against a head, logits never stored: l = h W^T + bias, then the row statistics of
// head_ops.cuh over the classes of every row.
#pragma once

#include "common.cuh"
#include "head_ops.cuh"

namespace lsam {

struct HeadArgs {
  int64_t rows, inner, classes, total;  // total = K * rows
  int64_t hk, hr, wk, wr, bk;  // strides: h worker / row, w worker / class, bias worker (the contraction index is contiguous)
  const float* bias;           // nullable
  const int32_t* labels;       // nullable
  int parts;                   // partial statistics per row
  int64_t per_split;           // SIMT form: classes of a block's share
  RowStat* part;               // [parts][K * rows]
  float* at_label;             // [K * rows] logit of the label
};

// Small products of any type, stride and size, on the FMA pipes: tiles of 32 rows x 128 classes x 16 inner indices, 256 threads with 2 x 8 outputs
// each.  A thread keeps the running statistics of its two rows over its columns of every tile of the block's share of the classes; the 16 threads
// of a row join at the end.  grid (shares, ceil(rows / 32), K)
constexpr int kHsM = 32, kHsN = 128, kHsK = 16;
template <typename T>
__global__ void __launch_bounds__(256)
head_score_simt_kernel(const T* __restrict__ h, const T* __restrict__ w, HeadArgs a) {
  __shared__ __align__(16) float hs[kHsK][kHsM + 4], wsm[kHsK][kHsN + 4];
  grid_dep_launch();  // the join may become resident; it waits for this grid
  const int64_t k = blockIdx.z, r0 = (int64_t)blockIdx.y * kHsM;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t c_begin = (int64_t)blockIdx.x * a.per_split, c_end = min(a.classes, c_begin + a.per_split);
  const T* hp = h + k * a.hk;
  const T* wp = w + k * a.wk;
  RowStat st[2];
  int32_t y[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    st[i] = stat_empty();
    const int64_t r = r0 + ty * 2 + i;
    y[i] = (a.labels && r < a.rows) ? a.labels[k * a.rows + r] : -1;
  }
  T x[10];  // 32 + 128 rows of 16, consecutive threads along the inner index: the next step's elements are on their way while this one's are used
  auto fetch = [&](int64_t c0, int64_t d0) {
#pragma unroll
    for (int q = 0; q < 10; ++q) {
      const int e = q * 256 + tid, rr = e >> 4;
      const int64_t d = d0 + (e & 15), r = q < 2 ? r0 + rr : c0 + rr - kHsM;
      x[q] = from_float<T>(0.f);
      if (d < a.inner && r < (q < 2 ? a.rows : c_end)) x[q] = q < 2 ? hp[r * a.hr + d] : wp[r * a.wr + d];
    }
  };
  fetch(c_begin, 0);
  for (int64_t c0 = c_begin; c0 < c_end; c0 += kHsN) {
    float acc[2][8] = {};
    for (int64_t d0 = 0; d0 < a.inner; d0 += kHsK) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 10; ++q) {
        const int e = q * 256 + tid, dd = e & 15, rr = e >> 4;
        if (q < 2) hs[dd][rr] = to_float(x[q]);
        else wsm[dd][rr - kHsM] = to_float(x[q]);
      }
      __syncthreads();
      if (d0 + kHsK < a.inner) fetch(c0, d0 + kHsK);
      else if (c0 + kHsN < c_end) fetch(c0 + kHsN, 0);
#pragma unroll
      for (int d = 0; d < kHsK; ++d) {
        const float4 b0 = *reinterpret_cast<const float4*>(&wsm[d][tx * 4]), b1 = *reinterpret_cast<const float4*>(&wsm[d][64 + tx * 4]);
        const float bv[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(hs[d][ty * 2 + i], bv[j], acc[i][j]);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t c = c0 + (j / 4) * 64 + tx * 4 + j % 4;
        if (c >= c_end) continue;
        const float l = acc[i][j] + (a.bias ? a.bias[k * a.bk + c] : 0.f);
        if (c == y[i]) a.at_label[k * a.rows + r0 + ty * 2 + i] = l;  // y is -1 in rows beyond the last
        stat_add(st[i], l);
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    for (int d = 8; d > 0; d >>= 1) st[i] = stat_merge(st[i], stat_shfl_xor(st[i], d));
    const int64_t r = r0 + ty * 2 + i;
    if (tx == 0 && r < a.rows) a.part[(int64_t)blockIdx.x * a.total + k * a.rows + r] = st[i];
  }
}

// Sums over the warp of N values a lane (N a power of two, at most 32): lane i ends with the sum of value sum_index<N>(i).  Halving: at every step a lane
// passes on the half it does not keep, so N values cost N - 1 exchanges instead of 5 N.
template <int N> __device__ inline int sum_index(int lane) {
  int v = 0;
#pragma unroll
  for (int b = 0, n = N; n > 1; ++b, n >>= 1) v += ((lane >> b) & 1) * (n >> 1);
  return v;
}
template <int N> __device__ inline float warp_sums(float (&v)[N], int lane) {
  int b = 0;
#pragma unroll
  for (int n = N; n > 1; n >>= 1, ++b) {
    const bool up = (lane >> b) & 1;
#pragma unroll
    for (int j = 0; j < n / 2; ++j) {
      const float keep = up ? v[j + n / 2] : v[j], pass = up ? v[j] : v[j + n / 2];
      v[j] = keep + __shfl_xor_sync(~0u, pass, 1 << b);
    }
  }
  for (; b < 5; ++b) v[0] += __shfl_xor_sync(~0u, v[0], 1 << b);
  return v[0];
}

// At most eight rows: the bytes of w bound the pass, and every element of w is used R times, so it goes straight from memory to the FMA pipes.  The R rows of
// h sit in shared memory as fp32; a warp takes G classes at a time, its lanes stride the inner index (16-byte vectors, or single elements where the
// rows of w are not aligned), R G products a lane and step; the lanes' sums meet by halving, which leaves a lane one logit.
// grid (shares, 1, K), block 256, shared memory gemv_smem
constexpr int kGemvRows = 8, kGemvSmem = 200 * 1024;
inline int64_t gemv_smem(int R, int64_t inner) { return (int64_t)R * round_up(inner, 256) * 4; }
template <typename T, int R, bool VEC>
__global__ void __launch_bounds__(256, 2)
head_gemv_kernel(const T* __restrict__ h, const T* __restrict__ w, HeadArgs a) {
  constexpr int G = R == 8 || (VEC && R == 4) ? 4 : 8, NV = R * G, N = VEC ? vec_n<T>() : 1;
  extern __shared__ __align__(16) float hs[];  // [R][inner rounded up to 256]
  __shared__ float red[3][8][NV];
  grid_dep_launch();
  const int64_t k = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int inner = (int)a.inner, hp = (int)round_up(a.inner, 256);
  // the order in which a lane reads h: vectors of eight are split so that both halves are read without bank conflicts
  auto place = [&](int d) { return N == 8 ? (d & ~255) + ((d >> 2) & 1) * 128 + ((d >> 3) & 31) * 4 + (d & 3) : d; };
  for (int e = tid; e < R * hp; e += 256) {
    const int r = e / hp, d = e % hp;
    hs[r * hp + place(d)] = r < a.rows && d < inner ? to_float(h[k * a.hk + r * a.hr + d]) : 0.f;
  }
  __syncthreads();
  const T* wp = w + k * a.wk;
  const int64_t c_begin = (int64_t)blockIdx.x * a.per_split, c_end = min(a.classes, c_begin + a.per_split);
  const int mine = sum_index<NV>(lane), row = mine % R, cls = mine / R;  // the value this lane ends with
  const bool owner = lane < NV && row < a.rows;
  const int32_t y = owner && a.labels ? a.labels[k * a.rows + row] : -1;
  RowStat st = stat_empty();
  for (int64_t c0 = c_begin + warp * G; c0 < c_end; c0 += 8 * G) {
    const T* p[G];
#pragma unroll
    for (int g = 0; g < G; ++g) p[g] = wp + min(c0 + g, c_end - 1) * a.wr;  // beyond the share: read again, not used
    float v[NV] = {};
    const int body = VEC ? inner / N * N : 0;
    if constexpr (VEC) {
#pragma unroll 2
      for (int d = lane * N; d < body; d += 32 * N) {
        uint4 x[G];
#pragma unroll
        for (int g = 0; g < G; ++g) x[g] = __ldg(reinterpret_cast<const uint4*>(p[g] + d));
        float hv[R][N];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int q = 0; q < N / 4; ++q) *reinterpret_cast<float4*>(&hv[r][4 * q]) = *reinterpret_cast<const float4*>(&hs[r * hp + place(d + 4 * q)]);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float f[N];
          vec_unpack<T>(x[g], f);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) v[g * R + r] = fmaf(f[j], hv[r][j], v[g * R + r]);
        }
      }
    }
    constexpr int S = VEC ? 1 : 4;  // single elements (all of them, or the last ones): S steps in flight
    for (int d = body + lane; d < inner; d += 32 * S) {
      float f[S][G];
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int g = 0; g < G; ++g) f[s][g] = d + 32 * s < inner ? to_float(p[g][d + 32 * s]) : 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float x = d + 32 * s < hp ? hs[r * hp + place(d + 32 * s)] : 0.f;
#pragma unroll
          for (int g = 0; g < G; ++g) v[g * R + r] = fmaf(f[s][g], x, v[g * R + r]);
        }
    }
    float l = warp_sums<NV>(v, lane);
    const int64_t c = c0 + cls;
    if (owner && c < c_end) {
      if (a.bias) l += a.bias[k * a.bk + c];
      if (c == y) a.at_label[k * a.rows + row] = l;
      stat_add(st, l);
    }
  }
  if (lane < NV) { red[0][warp][mine] = st.m; red[1][warp][mine] = st.s; red[2][warp][mine] = st.t; }
  __syncthreads();
  if (warp < R && warp < a.rows) {  // warp r joins row r: 8 warps x G lanes
    RowStat t = stat_empty();
    for (int e = lane; e < 8 * G; e += 32) {
      const int q = e / G, m = (e % G) * R + warp;
      t = stat_merge(t, RowStat{red[0][q][m], red[1][q][m], red[2][q][m]});
    }
    t = warp_stat(t);
    if (lane == 0) a.part[(int64_t)blockIdx.x * a.total + k * a.rows + warp] = t;
  }
}

// Copies h and w, [Z][rows][inner] of any strides, into rows of `pad` elements (a multiple of 8) that TMA takes, in one launch.  fp32 is split into three
// bf16 planes p0 = bf16(x), p1 = bf16(x - p0), p2 = bf16(x - p0 - p1), [3][Z][rows][pad], whose sum is x; 16-bit types keep theirs.  `lanes` (a power of
// two) consecutive threads move consecutive elements of a row; a block walks the rows, kCopyRows of a thread in flight.
// Bound by the bytes and, for 16-bit elements moved one by one, by issue.  Measured (us of the whole call): 2000 x 1021 x 16384 bf16 96 (one row in flight and
// a launch for each matrix 98), 16 x 1091 x 1000 13.9 (17.4), 4 x 128 x 1078 x 3688 fp32 93 (94); eight rows in flight 118, 16.4, 100.
// grid h.blocks + w.blocks, block 256; a side's blocks: column block fastest, then row block, then worker
constexpr int kCopyRows = 4;
struct CopySide {
  const void* src;
  void* dst;
  int64_t sk, sr, rows, Z;
  uint32_t row_blocks, blocks;
};
template <typename T, typename D>
__global__ void __launch_bounds__(256, 6)
head_copy_kernel(CopySide h, CopySide w, int64_t inner, int64_t pad, int lanes, uint32_t cols) {
  constexpr int U = kCopyRows;
  const bool first = blockIdx.x < h.blocks;
  const CopySide a = first ? h : w;
  const uint32_t b = first ? blockIdx.x : blockIdx.x - h.blocks;
  const int64_t d = (int64_t)(b % cols) * lanes + (threadIdx.x & (lanes - 1)), k = b / cols / a.row_blocks;
  if (d >= inner) return;
  const int group = 256 / lanes;
  const int64_t plane = a.Z * a.rows * pad, step = (int64_t)a.row_blocks * group;
  const T* __restrict__ src = static_cast<const T*>(a.src) + k * a.sk + d;
  D* __restrict__ dst = static_cast<D*>(a.dst) + k * a.rows * pad + d;
  for (int64_t r = (int64_t)(b / cols % a.row_blocks) * group + threadIdx.x / lanes; r < a.rows; r += U * step) {
    T x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r + u * step < a.rows) x[u] = __ldg(src + (r + u * step) * a.sr);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r + u * step >= a.rows) break;
      D* p = dst + (r + u * step) * pad;
      if constexpr (sizeof(T) == 4) {
        float f = to_float(x[u]);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          const D v = from_float<D>(f);
          p[q * plane] = v;
          f -= to_float(v);
        }
      } else {
        *p = x[u];
      }
    }
  }
}

// Joins the partial statistics of a row in a fixed order: a warp per row, lane i takes partials i, i + 32, ..., then the lanes meet.
// grid ceil(total / 8), block 256
__global__ void __launch_bounds__(256)
head_join_kernel(HeadArgs a, int64_t total, ScoreOut o) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= total) return;
  RowStat st = stat_empty();
#pragma unroll 4
  for (int p = lane; p < a.parts; p += 32) st = stat_merge(st, a.part[(int64_t)p * total + r]);
  st = warp_stat(st);
  if (lane != 0) return;
  const int32_t y = a.labels ? a.labels[r] : 0;
  float lse = 0.f, ent = 0.f, lp = 0.f;
  if (y >= 0) {
    const RowScore sc = stat_finish(st);
    lse = sc.lse;
    ent = sc.ent;
    if (o.logp) lp = y < a.classes ? score_logp(a.at_label[r], sc) : NAN;
  }
  if (o.logp) o.logp[r] = lp;
  if (o.lse) o.lse[r] = lse;
  if (o.entropy) o.entropy[r] = ent;
}

}  // namespace lsam
