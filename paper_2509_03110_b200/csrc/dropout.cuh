// dropout.cuh -- dropout whose mask is a function of (seed, tick, layer, worker, row, column) and is never stored.
//
// One Philox4x32-10 block gives the 16-bit numbers of eight columns: the generator's twenty wide multiplications cost about five instructions
// per element, little enough that the bytes of x, skip and out bound the pass (with 32-bit numbers, four columns a block, it would be ten).
#pragma once

#include "common.cuh"
#include "head_ops.cuh"

namespace lsam {

struct DropArgs {
  int64_t rows, n;
  int64_t xk, xr, sk, sr, ok, orr;  // strides of x, skip and out: worker, row (columns are contiguous)
  uint32_t key0, key1, tick, word2; // Philox key; counter words 3 and 2 (the latter for worker 0)
  uint32_t limit;                   // an element is dropped when its 16 bits, moved to the top of a word, are below `limit`
  bool some;                        // false: everything is dropped
  float scale;                      // 65536 / (65536 - cut)
  FastDiv by_groups, by_rows;       // by_groups: groups of 8 (vector form) or segments of 256 columns per row
  __device__ inline void bits(uint32_t k, uint32_t r, uint32_t g, uint32_t (&w)[4]) const {  // columns 8 g .. 8 g + 7
    philox4x32_10(g, r, word2 + k, tick, key0, key1, w);
  }
  // `top`: the element's 16 bits at the top of a word; what lies below them does not reach the comparison
  __device__ inline float value(float x, uint32_t top) const { return some && top >= limit ? x * scale : 0.f; }
};

constexpr int kDropUnroll = 2;

// Every row starts on a 16-byte boundary: a thread owns kDropUnroll groups of eight columns (one 16-byte vector of each tensor, two in fp32); a row's
// last columns, when they are no whole group, move one by one.
template <typename T>
__global__ void __launch_bounds__(256)
dropout_vec_kernel(const T* x, const T* skip, T* out, DropArgs a, uint32_t total) {
  constexpr int NV = (int)sizeof(T) / 2, N = vec_n<T>();  // vectors per group
#pragma unroll
  for (int u = 0; u < kDropUnroll; ++u) {
    const uint32_t e = (blockIdx.x * kDropUnroll + u) * 256u + threadIdx.x;
    if (e >= total) return;
    uint32_t g, r;
    const uint32_t k = a.by_rows.div(a.by_groups.div(e, g), r);
    const int64_t c = (int64_t)g * 8;
    const T* xp = x + k * a.xk + r * a.xr + c;
    const T* sp = skip ? skip + k * a.sk + r * a.sr + c : nullptr;
    T* op = out + k * a.ok + r * a.orr + c;
    uint32_t w[4];
    if (c + 8 <= a.n) {
      uint4 xv[NV], sv[NV];
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        xv[q] = reinterpret_cast<const uint4*>(xp)[q];
        if (sp) sv[q] = reinterpret_cast<const uint4*>(sp)[q];
      }
      a.bits(k, r, g, w);
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        float v[N];
        vec_unpack<T>(xv[q], v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int b = q * N + j;
          v[j] = a.value(v[j], (b & 1) ? w[b >> 1] : w[b >> 1] << 16);
        }
        if (sp) {
          float s[N];
          vec_unpack<T>(sv[q], s);
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] += s[j];
        }
        reinterpret_cast<uint4*>(op)[q] = vec_pack<T>(v);
      }
    } else {
      a.bits(k, r, g, w);
#pragma unroll
      for (int b = 0; b < 8; ++b)
        if (c + b < a.n) {
          float v = a.value(to_float(xp[b]), (b & 1) ? w[b >> 1] : w[b >> 1] << 16);
          if (sp) v += to_float(sp[b]);
          op[b] = from_float<T>(v);
        }
    }
  }
}

// Any alignment: a warp takes 256 columns of a row.  Lane i draws the numbers of its group of eight and leaves them in shared memory, so that
// consecutive lanes move consecutive elements.
template <typename T>
__global__ void __launch_bounds__(256)
dropout_elem_kernel(const T* x, const T* skip, T* out, DropArgs a, uint32_t total) {
  __shared__ __align__(16) uint16_t num[8][256];
  const int wp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * 8 + wp;
  if (unit >= total) return;
  uint32_t seg, r;
  const uint32_t k = a.by_rows.div(a.by_groups.div(unit, seg), r);
  const int64_t c0 = (int64_t)seg * 256 + lane;
  const int n = c0 < a.n ? (int)min((int64_t)8, (a.n - c0 + 31) / 32) : 0;  // this lane's columns
  const T* xp = x + k * a.xk + r * a.xr + c0;
  const T* sp = skip ? skip + k * a.sk + r * a.sr + c0 : nullptr;
  T* op = out + k * a.ok + r * a.orr + c0;
  float v[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = e < n ? to_float(xp[e * 32]) : 0.f;
    s[e] = e < n && sp ? to_float(sp[e * 32]) : 0.f;
  }
  uint32_t w[4];
  a.bits(k, r, seg * 32 + lane, w);
  *reinterpret_cast<uint4*>(&num[wp][lane * 8]) = make_uint4(w[0], w[1], w[2], w[3]);
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) {
      float y = a.value(v[e], (uint32_t)num[wp][lane + e * 32] << 16);
      if (sp) y += s[e];
      op[e * 32] = from_float<T>(y);
    }
}

}  // namespace lsam
