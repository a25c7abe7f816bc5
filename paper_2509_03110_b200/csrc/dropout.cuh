// dropout.cuh -- dropout whose mask is a function of (seed, tick, layer, worker, row, column) and is never stored.
#pragma once

#include "common.cuh"

namespace lsam {

struct DropArgs {
  int64_t rows, n;
  int64_t xk, xr, sk, sr, ok, orr;  // strides of x, skip and out: worker, row (columns are contiguous)
  uint32_t key0, key1, tick, word2; // Philox key; counter words 3 and 2 (the latter for worker 0)
  uint32_t cut;                     // an element is dropped when its 16 bits are below `cut`
  float scale;                      // 65536 / (65536 - cut)
};

// The 16 random bits of the eight columns 8 g .. 8 g + 7 of a row: word j / 2 of the Philox block, low half first.
__device__ inline void drop_bits(const DropArgs& a, int64_t k, int64_t r, int64_t g, uint32_t (&w)[4]) {
  philox4x32_10((uint32_t)g, (uint32_t)r, a.word2 + (uint32_t)k, a.tick, a.key0, a.key1, w);
}

// out = skip + (kept ? x * scale : 0); one thread per group of eight columns
template <typename T>
__global__ void __launch_bounds__(256)
dropout_kernel(const T* x, const T* skip, T* out, DropArgs a, int64_t groups, int64_t total) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  const int64_t g = e % groups, kr = e / groups, r = kr % a.rows, k = kr / a.rows;
  uint32_t w[4];
  drop_bits(a, k, r, g, w);
  for (int j = 0; j < 8; ++j) {
    const int64_t c = g * 8 + j;
    if (c >= a.n) break;
    const uint32_t bits = (w[j >> 1] >> (16 * (j & 1))) & 0xffffu;
    float y = bits >= a.cut ? to_float(x[k * a.xk + r * a.xr + c]) * a.scale : 0.f;
    if (skip) y += to_float(skip[k * a.sk + r * a.sr + c]);
    out[k * a.ok + r * a.orr + c] = from_float<T>(y);
  }
}

}  // namespace lsam
