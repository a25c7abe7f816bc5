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

constexpr int kHsM = 64, kHsN = 64, kHsK = 16;  // rows, classes and contraction of a tile

// Any type, any stride, any size: 64 x 64 tiles of fp32 products, 256 threads with 4 x 4 outputs each.  A thread keeps the running
// statistics of its four rows over its columns of every tile of the share; the 16 threads of a row join at the end.
// grid (splits, ceil(rows / 64), K)
template <typename T>
__global__ void __launch_bounds__(256)
head_score_simt_kernel(const T* __restrict__ h, const T* __restrict__ w, HeadArgs a) {
  __shared__ float hs[kHsK][kHsM + 4], wsm[kHsK][kHsN + 4];
  grid_dep_launch();  // the join may become resident; it waits for this grid
  const int64_t k = blockIdx.z, r0 = (int64_t)blockIdx.y * kHsM;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t c_begin = (int64_t)blockIdx.x * a.per_split, c_end = min(a.classes, c_begin + a.per_split);
  const T* hp = h + k * a.hk;
  const T* wp = w + k * a.wk;
  RowStat st[4];
  int32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    st[i] = stat_empty();
    const int64_t r = r0 + ty * 4 + i;
    y[i] = (a.labels && r < a.rows) ? a.labels[k * a.rows + r] : -1;
  }
  for (int64_t c0 = c_begin; c0 < c_end; c0 += kHsN) {
    float acc[4][4] = {};
    for (int64_t d0 = 0; d0 < a.inner; d0 += kHsK) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = q * 256 + tid, rr = e >> 4, dd = e & 15;
        hs[dd][rr] = (r0 + rr < a.rows && d0 + dd < a.inner) ? to_float(hp[(r0 + rr) * a.hr + d0 + dd]) : 0.f;
        wsm[dd][rr] = (c0 + rr < c_end && d0 + dd < a.inner) ? to_float(wp[(c0 + rr) * a.wr + d0 + dd]) : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int d = 0; d < kHsK; ++d) {
        const float4 hv = *reinterpret_cast<const float4*>(&hs[d][ty * 4]);
        const float4 wv = *reinterpret_cast<const float4*>(&wsm[d][tx * 4]);
        const float ha[4] = {hv.x, hv.y, hv.z, hv.w}, wa[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(ha[i], wa[j], acc[i][j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t c = c0 + tx * 4 + j;
      if (c >= c_end) break;
      const float b = a.bias ? a.bias[k * a.bk + c] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float l = acc[i][j] + b;
        stat_add(st[i], l);
        if (c == y[i]) a.at_label[k * a.rows + r0 + ty * 4 + i] = l;  // y is -1 in rows beyond the last
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    for (int d = 8; d > 0; d >>= 1) st[i] = stat_merge(st[i], stat_shfl_xor(st[i], d));
    const int64_t r = r0 + ty * 4 + i;
    if (tx == 0 && r < a.rows) a.part[((int64_t)blockIdx.x * gridDim.z + k) * a.rows + r] = st[i];
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
