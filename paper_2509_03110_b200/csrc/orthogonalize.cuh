// orthogonalize.cuh -- a matrix made nearly orthogonal by Newton-Schulz products on the 5th-generation tensor cores.
//
//   X_0 = G / (|G|_F + eps);   X_{t+1} = a X_t + (b A + c A^2) X_t,  A = X_t X_t^T;   result scale * X_steps
// An odd polynomial of the singular values, the same one at every step, that moves all of them towards one.  G is taken with its smaller side as rows, m <= n
// (a tall matrix is transposed on its way in and out), so A is m x m.  Three products a step:
//   GRAM    A = X X^T           m^2 n multiply-adds, half of them: tiles below the diagonal are written by those above, transposed
//   SQUARE  P = b A + c A A     m^3, half of them likewise (A = A^T, so both operands are read along their rows)
//   APPLY   X' = a X + P X      m^2 n; X is read with its columns contiguous (the N-contiguous form of the B operand), so no transposed copy is kept
//
// Numbers.  Every matrix is held as two fp16 planes hi + lo, hi = fp16(2^e x), lo = fp16(2^e x - hi), e a power of two for the whole matrix, chosen by the host
// from the largest singular value that the polynomial allows at that step (no element can be larger): 2^-24 of an element down to 2^-16 of that bound, 2^-40 of the bound
// below.  A product takes three products of planes, hi hi + lo hi + hi lo, what is left out being 2^-24 of each term: fp32 accuracy for half of what three
// bf16 planes and six products cost.  The tensor core cuts off what lies below the accumulator's last place at each step of 16 inner indices, so sums
// go in chunks of kNsChunk blocks of 64 indices, the small products of a block first, and the chunks are added in registers (8 x 1024 x 784 fp32, error against 64 bits and
// time: one block 1.5e-6, 566 us; two 3.1e-6 or more, 550; a plain fp32 chain 2.8e-6).
// The type that the result is stored in changes nothing of that: what an error grows to depends on how the norm of G is spread over its directions, on the
// coefficients and on the steps.  With hi hi alone in most places (2 x 4096 x 4096 bf16 in 3.2 instead of 7.2 ms) a dense result of 512 rows was off by 1.2e-3 of its norm after
// five steps (rounding to bf16: 1.7e-3), but one of eight rows that hold all of the norm by 8e-3, and with (4.0848, -6.8946, 2.9270) by 6e-2; with 512 indices in an
// accumulator (6.3 ms) a dense fp16 result was off by about 1e-4 after ten steps (rounding: 2e-4; this form and the fp32 chain: 1e-5).
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "tc_ptx.cuh"
#include "vec.cuh"

namespace lsam {

// ------------------------------------------------------------------------------------------------ norm and start
// Partial sums of squares, in double: g^2 of fp32 leaves the fp32 range.  grid (chunks, K); unit e of a worker: (e / inner, e % inner), the inner index the
// one of the smaller stride; a unit is an element, or (VEC) the 16-byte vector of a contiguous index (2 x 4096 x 4096 bf16: 77 us by
// elements, 25 by vectors).
constexpr int kNsNorm = 4096;  // elements of a partial sum, a multiple of this
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
ns_norm_kernel(const T* g, int64_t sk, int64_t so, int64_t si, int64_t inner, int64_t total, int64_t chunk, double* part) {
  constexpr int N = VEC ? vec_n<T>() : 1, AHEAD = VEC ? 4 : 16;
  using Raw = typename std::conditional<VEC, uint4, T>::type;
  __shared__ double smem[8];
  grid_dep_launch();
  const int64_t e0 = (int64_t)blockIdx.x * chunk, e1 = min(total, e0 + chunk);
  g += blockIdx.y * sk;
  double s = 0.0;
  // 32-bit division where it does
  const int64_t at = e0 + threadIdx.x;
  int64_t o = total < ((int64_t)1 << 32) ? (int64_t)((uint32_t)at / (uint32_t)inner) : at / inner, i = at - o * inner;
  const int64_t step_o = 256u / (uint32_t)inner, step_i = 256u % (uint32_t)inner;
  for (int64_t e = e0 + threadIdx.x; e < e1; e += 256 * AHEAD) {
    Raw v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const bool have = e + u * 256 < e1;
      if constexpr (VEC) v[u] = have ? *reinterpret_cast<const uint4*>(g + o * so + i * N) : make_uint4(0u, 0u, 0u, 0u);
      else v[u] = have ? g[o * so + i * si] : from_float<T>(0.f);
      o += step_o;
      i += step_i;
      if (i >= inner) { i -= inner; ++o; }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      float f[N];
      if constexpr (VEC) vec_unpack<T>(v[u], f);
      else f[0] = to_float(v[u]);
#pragma unroll
      for (int q = 0; q < N; ++q) s = fma((double)f[q], (double)f[q], s);
    }
  }
  s = block_sum(s, smem);
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}
// 1 / (|G| + eps) of |G|^2 = s; NaN, not 0, where an element is infinite
__device__ inline double ns_inverse_of(double s, double eps) { return isinf(s) ? (double)NAN : 1.0 / (sqrt(s) + eps); }
// The same of partial sums, in a fixed order, in every thread of a block of 256
__device__ inline double ns_inverse(const double* part, int chunks, float eps) {
  __shared__ double smem[9];
  double s = 0.0;
  for (int c = threadIdx.x; c < chunks; c += 256) s += part[c];
  s = block_sum(s, smem);
  if (threadIdx.x == 0) smem[8] = s;
  __syncthreads();
  return ns_inverse_of(smem[8], (double)eps);
}

__device__ inline void ns_split(float v, fp16& hi, fp16& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}
__device__ inline void ns_split2(float v, float w, __half2& hi, __half2& lo) {  // two at a time: a conversion for both
  hi = __floats2half2_rn(v, w);
  const float2 f = __half22float2(hi);
  lo = __floats2half2_rn(v - f.x, w - f.y);
}
// One matrix per worker as planes: hi at p + k 2 plane, lo at p + (2 k + 1) plane, rows ld apart.
struct NsPlanes {
  fp16* p;
  int64_t plane, ld;
};

// X_0 [m][n] from G, element (i, j) at i si + j sj.  Tiles of 64 x 64 through shared memory, read along the smaller stride and written along j.
template <typename T>
__global__ void __launch_bounds__(256, 4)
ns_start_kernel(const T* g, int64_t sk, int64_t si, int64_t sj, int64_t m, int64_t n, const double* part, int chunks, float eps, double scale, NsPlanes x) {
  __shared__ float tile[64][65];
  grid_dep_sync();
  const int64_t i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
  const int k = blockIdx.z;
  const T* p = g + k * sk;
  // rows u, u + 4, ... of the tile in the order in which it is read, column v
  const bool rows = sj <= si;
  const int u = threadIdx.x >> 6, v = threadIdx.x & 63;
  const int64_t su = rows ? si : sj, left = (rows ? m - i0 : n - j0) - u;
  const bool have = v < (rows ? n - j0 : m - i0);
  p += (i0 + (rows ? u : v)) * si + (j0 + (rows ? v : u)) * sj;
  T f[16];
#pragma unroll
  for (int q = 0; q < 16; ++q) f[q] = have && 4 * q < left ? p[4 * q * su] : from_float<T>(0.f);
  const double inv = ns_inverse(part + (int64_t)k * chunks, chunks, eps) * scale;
  float* to = rows ? &tile[u][v] : &tile[v][u];
#pragma unroll
  for (int q = 0; q < 16; ++q) to[4 * q * (rows ? 65 : 1)] = (float)((double)to_float(f[q]) * inv);
  __syncthreads();
  fp16* hi = x.p + (int64_t)k * 2 * x.plane;
  for (int e = threadIdx.x; e < 512; e += 256) {
    const int i = e >> 3, j = (e & 7) * 8;
    if (i0 + i >= m || j0 + j >= x.ld) continue;
    union { uint4 q; fp16 h[8]; } a, b;
#pragma unroll
    for (int u = 0; u < 8; ++u) ns_split(tile[i][j + u], a.h[u], b.h[u]);
    const int64_t at = (i0 + i) * x.ld + j0 + j;
    *reinterpret_cast<uint4*>(hi + at) = a.q;
    *reinterpret_cast<uint4*>(hi + x.plane + at) = b.q;
  }
}

// The same where rows of G are contiguous and hold whole vectors of eight: eight columns a thread, no tile (2 x 4096 x 4096 bf16: 84 -> 44 us).
template <typename T>
__global__ void __launch_bounds__(256)
ns_start_rows_kernel(const T* g, int64_t sk, int64_t si, uint32_t groups, int64_t total, const double* part, int chunks, float eps, double scale, NsPlanes x) {
  constexpr int N = vec_n<T>();
  grid_dep_sync();
  const int k = blockIdx.y;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = total < ((int64_t)1 << 32) ? (int64_t)((uint32_t)e / groups) : e / groups, j = (e - i * groups) * 8;
  uint4 q[8 / N];
#pragma unroll
  for (int u = 0; u < 8 / N; ++u) q[u] = e < total ? reinterpret_cast<const uint4*>(g + k * sk + i * si + j)[u] : make_uint4(0u, 0u, 0u, 0u);
  const double inv = ns_inverse(part + (int64_t)k * chunks, chunks, eps) * scale;
  if (e >= total) return;
  union { uint4 q4; __half2 h[4]; } a, b;
#pragma unroll
  for (int u = 0; u < 8 / N; ++u) {
    float f[N];
    vec_unpack<T>(q[u], f);
#pragma unroll
    for (int w = 0; w < N; w += 2) ns_split2((float)((double)f[w] * inv), (float)((double)f[w + 1] * inv), a.h[(u * N + w) / 2], b.h[(u * N + w) / 2]);
  }
  fp16* hi = x.p + (int64_t)k * 2 * x.plane + i * x.ld + j;
  *reinterpret_cast<uint4*>(hi) = a.q4;
  *reinterpret_cast<uint4*>(hi + x.plane) = b.q4;
}

// No steps: out = scale X_0.
template <typename T>
__global__ void __launch_bounds__(256)
ns_only_norm_kernel(const T* g, int64_t sk, int64_t si, int64_t sj, int64_t m, int64_t n, const double* part, int chunks, float eps, float scale, T* out, int64_t ok, int64_t oi, int64_t oj) {
  const double inv = ns_inverse(part + (int64_t)blockIdx.y * chunks, chunks, eps) * (double)scale;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= m * n) return;
  const int64_t i = e / n, j = e - i * n;
  out[blockIdx.y * ok + i * oi + j * oj] = from_float<T>((float)((double)to_float(g[blockIdx.y * sk + i * si + j * sj]) * inv));
}

// ------------------------------------------------------------------------------------------------ products
constexpr int kNsThreads = 384;  // warp 0: TMA, warp 1: MMA and tensor memory, warps 4-11: draining (two per quadrant of lanes)
constexpr int kNsRegsIssue = 56, kNsRegsDrain = 216;
static_assert((kNsRegsIssue + 2 * kNsRegsDrain) * 128 <= 168 * kNsThreads, "setmaxnreg draws on the registers of the launch");
constexpr int kNsK = 64;
constexpr int kNsChunk = 1;  // blocks of 64 inner indices that share an accumulator
constexpr int kNsMaxStages = 8, kNsRing = 192 * 1024, kNsSmem = kNsRing + 8 * 4096 + 1024 + 256;

enum : int { NS_GRAM = 0, NS_SQUARE = 1, NS_APPLY = 2, NS_FINAL = 3, NS_PART = 4 };  // NS_PART: a share of a Gram matrix's inner indices, in fp32

struct NsGemm {
  int m, n, inner;        // of the product
  int tile_n, m_tiles, n_tiles;
  int stages, stage_bytes, a_bytes, b_bytes;
  uint32_t idesc;
  int sym;                // a symmetric result: tiles below the diagonal are the transposed ones above
  int splits, split_blocks;  // NS_PART: shares of the inner indices, blocks of 64 of a share (else 1 and all)
  int64_t per_k, units;   // tiles of a worker (of a share of one), of all
  float f, h, diagonal;   // result = f * product; NS_SQUARE: + h * (hi + lo of `other`) + diagonal * I
  NsPlanes other, out;    // the same sizes; `out`: not NS_FINAL
  void* final_out;        // NS_FINAL
  int64_t ok, oi, oj;
};
// Tiles are numbered row by row; a symmetric result has those with a column at or behind the diagonal.  k: worker * splits + share.
template <bool SYM, int TM>
__device__ inline void ns_tile(const NsGemm& g, int64_t u, int& k, int& mt, int& nt) {
  k = (int)(u / g.per_k);
  int r = (int)(u - (int64_t)k * g.per_k);
  mt = 0;
  if (SYM && g.sym) {
    for (;; ++mt) {
      const int first = mt * TM / g.tile_n, have = g.n_tiles - first;
      if (r < have) { nt = first + r; return; }
      r -= have;
    }
  } else {
    mt = r / g.n_tiles;
    nt = r - mt * g.n_tiles;
  }
}

// A warp's blocks of 32 rows x 32 columns go between registers (a lane its row) and memory through 2 KB of shared memory a plane, rows of 64 bytes in the 64-byte
// swizzle of the tensor maps (16-byte piece q of row r at q ^ (r / 2 % 4)): a lane by itself would touch one row of 32 in every access.
__device__ __forceinline__ uint4* ns_piece(uint8_t* stage, int row, int q) { return reinterpret_cast<uint4*>(stage + row * 64 + ((q ^ (row >> 1)) & 3) * 16); }
// v += h (hi + lo) of rows i0 .. and columns c ..: eight rows an access, 64 bytes of each
__device__ __forceinline__ void ns_add_planes(float (&v)[32], float h, const fp16* p, int64_t plane, int64_t ld, int64_t i0, int64_t m, int64_t c, uint8_t* stage, int lane) {
  const int q = lane & 3, r0 = lane >> 2;
  uint4 w[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + r0 + 8 * u, col = c + 8 * q;
      w[t][u] = i < m && col < ld ? *reinterpret_cast<const uint4*>(p + t * plane + i * ld + col) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) *ns_piece(stage + t * 2048, r0 + 8 * u, q) = w[t][u];
  __syncwarp();
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    union { uint4 q4; __half2 h2[4]; } a, b;
    a.q4 = *ns_piece(stage, lane, u);
    b.q4 = *ns_piece(stage + 2048, lane, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = __half22float2(a.h2[e]), y = __half22float2(b.h2[e]);
      v[8 * u + 2 * e] = fmaf(h, x.x + y.x, v[8 * u + 2 * e]);
      v[8 * u + 2 * e + 1] = fmaf(h, x.y + y.y, v[8 * u + 2 * e + 1]);
    }
  }
  __syncwarp();
}
// As planes, by two copies of the bulk engine (what lies outside the matrix is clipped).
__device__ __forceinline__ void ns_store_planes(const float (&v)[32], const CUtensorMap* map, int k, int i0, int c, uint8_t* stage, int lane) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    union { uint4 q4; __half2 h[4]; } a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) ns_split2(v[8 * u + 2 * e], v[8 * u + 2 * e + 1], a.h[e], b.h[e]);
    *ns_piece(stage, lane, u) = a.q4;
    *ns_piece(stage + 2048, lane, u) = b.q4;
  }
  tc::fence_proxy_async();
  __syncwarp();
  if (lane == 0) {
    tc::tma_store_3d(map, stage, c, i0, 2 * k);
    tc::tma_store_3d(map, stage + 2048, c, i0, 2 * k + 1);
    tc::bulk_commit();
  }
}
__device__ __forceinline__ void ns_stage_free(int lane) {  // the copies have read the warp's shared memory
  if (lane == 0) tc::bulk_wait_read<0>();
  __syncwarp();
}
// The block that ns_store_planes has left in shared memory, transposed: its column j is row j0 + j of the output, columns i0 ...  ldmatrix turns 8 x 8 pieces.
__device__ __forceinline__ void ns_store_mirror(const uint8_t* stage, fp16* hi, int64_t plane, int64_t ld, int64_t i0, int64_t j0, int64_t n, int lane) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t r[4];
      const uint32_t at = tc::smem_u32(ns_piece(const_cast<uint8_t*>(stage) + t * 2048, lane, q));  // lane 8 e + f: row f of piece e
      asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
      fp16* to = hi + t * plane + (j0 + 8 * q + (lane >> 2)) * ld + i0 + 2 * (lane & 3);
      const int left = j0 + 8 * q + (lane >> 2) < n ? (int)min((int64_t)32, n - i0) - 2 * (lane & 3) : 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (8 * e < left) *reinterpret_cast<uint32_t*>(to + 8 * e) = r[e];  // ld is even: a pair may end in the padding
    }
  __syncwarp();
}
// The result: along its columns (a transposed matrix: lanes are neighbours there already), or a row at a time through shared memory.
template <typename T>
__device__ __forceinline__ void ns_store_final(const float (&v)[32], const NsGemm& g, int k, int64_t i0, int64_t c, float* stage, int lane) {
  T* to = static_cast<T*>(g.final_out) + k * g.ok;
  const int rows = (int)min((int64_t)32, g.m - i0), cols = (int)min((int64_t)32, g.n - c);
  if (g.oi == 1 && g.oj != 1) {
    if (lane < rows) {
      T* p = to + i0 + lane + c * g.oj;
#pragma unroll
      for (int j = 0; j < 32; ++j, p += g.oj)
        if (j < cols) *p = from_float<T>(v[j]);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 32; ++j) stage[lane * 32 + (j ^ lane)] = v[j];
  __syncwarp();
  if (lane < cols) {
    T* p = to + i0 * g.oi + (c + lane) * g.oj;
#pragma unroll 4
    for (int r = 0; r < rows; ++r, p += g.oi) *p = from_float<T>(stage[r * 32 + (lane ^ r)]);
  }
  __syncwarp();
}

// grid: CTAs (PAIR: clusters of 2 that share a tile of 256 rows, cta_group::2), each walking tiles u, u + grid, ...
// A stage holds 64 inner indices of every plane: [A hi, lo][B hi, lo].  All waits are bounded; a CTA that gives up leaves NaN in its tiles.
// STARVED (self-test): no operand is ever copied and the waits are short, so all of them run out with nothing in flight.
template <typename T, int EPI, bool PAIR, bool STARVED>
__global__ void __launch_bounds__(kNsThreads, 1)
ns_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out, const NsGemm g) {
  constexpr bool SYM = EPI == NS_GRAM || EPI == NS_SQUARE, B_MN = EPI == NS_APPLY || EPI == NS_FINAL, WHOLE = EPI == NS_FINAL || EPI == NS_PART;  // WHOLE: no planes
  constexpr int TM = PAIR ? 256 : 128;
  constexpr uint32_t LIMIT = STARVED ? 1u << 13 : tc::kSpinLimit;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* stages = ring + kNsRing;  // [8 draining warps][4 KB]
  uint64_t* full = reinterpret_cast<uint64_t*>(stages + 8 * 4096);  // [stages]
  uint64_t* empty = full + kNsMaxStages;
  uint64_t* acc_full = empty + kNsMaxStages;  // [4]
  uint64_t* acc_empty = acc_full + 4;         // [4]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kNsMaxStages + 8) * 8 + 8 <= 256 && kNsSmem <= 227 * 1024, "barrier area");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? tc::cluster_ctarank() : 0u;
  const bool leader = rank == 0u;
  const int64_t unit = PAIR ? blockIdx.x / 2 : blockIdx.x, units = PAIR ? gridDim.x / 2 : gridDim.x;
  const int k_blocks = (g.inner + kNsK - 1) / kNsK;
  // blocks of 64 inner indices of a unit: all, or its share
  const auto first_block = [&](int k) { return EPI == NS_PART ? k % g.splits * g.split_blocks : 0; };
  const auto end_block = [&](int k) { return EPI == NS_PART ? min(k_blocks, first_block(k) + g.split_blocks) : k_blocks; };
  const int b_rows = PAIR ? g.tile_n / 2 : g.tile_n;  // columns of the tile staged by this CTA

  grid_dep_launch();
  if (threadIdx.x == 0) {
    tc::prefetch_tensormap(&map_a);
    tc::prefetch_tensormap(&map_b);
    tc::prefetch_tensormap(&map_out);
    for (int s = 0; s < g.stages; ++s) { tc::mbar_init(&full[s], 1); tc::mbar_init(&empty[s], 1); }
    for (int s = 0; s < 4; ++s) { tc::mbar_init(&acc_full[s], 1); tc::mbar_init(&acc_empty[s], PAIR ? 16 : 8); }
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    if (PAIR) tc::tmem_alloc_pair(tmem_slot, 512);
    else tc::tmem_alloc(tmem_slot, 512);
  }
  tc::tc_fence_before();
  __syncthreads();
  if (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after();
  grid_dep_wait();
  const uint32_t tmem_base = *tmem_slot;
  // accumulators: what the products can be ahead of a tile's end, two of 256 columns or four
  const int accs = g.tile_n <= 128 ? 4 : 2;
  const uint32_t acc_cols = 512u / accs;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kNsRegsIssue));
    const bool one = ht_elect();
    if (!STARVED && warp == 0 && (PAIR || one)) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      const uint32_t ring0 = tc::smem_u32(ring), full0 = tc::smem_u32(full), empty0 = tc::smem_u32(empty);
      const uint32_t bar0 = PAIR ? tc::map_to_cta(full0, 0u) : full0;
      const uint32_t tx = (PAIR ? 2u : 1u) * (uint32_t)g.stage_bytes;
      for (int64_t u = unit; u < g.units && ok; u += units) {
        int k, mt, nt;
        ns_tile<SYM, TM>(g, u, k, mt, nt);
        const int r0 = mt * TM + (int)rank * 128, c0 = nt * g.tile_n + (int)rank * b_rows, kb1 = end_block(k), z = 2 * (EPI == NS_PART ? k / g.splits : k);
        for (int kb = first_block(k); kb < kb1; ++kb) {
          if (!ht_wait<LIMIT>(empty0 + 8 * s, ph ^ 1u, abort_flag)) { ok = false; break; }
          uint32_t dst = ring0 + s * g.stage_bytes;
          const uint32_t bar = bar0 + 8 * s;
          if (!PAIR || one) {
            if (!PAIR || leader) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full0 + 8 * s), "r"(tx) : "memory");
            for (int p = 0; p < 2; ++p, dst += g.a_bytes) ht_load<PAIR>(dst, &map_a, kb * kNsK, r0, z + p, bar);
            for (int p = 0; p < 2; ++p, dst += g.b_bytes) {
              if (B_MN) {
                for (int i = 0; i < b_rows / 64; ++i) ht_load<PAIR>(dst + i * 8192, &map_b, c0 + 64 * i, kb * kNsK, z + p, bar);
              } else {
                ht_load<PAIR>(dst, &map_b, kb * kNsK, c0, z + p, bar);
              }
            }
          }
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) *abort_flag = 1;
    }
    if (warp == 1 && leader && (PAIR || one)) {
      int s = 0, as = 0;
      uint32_t ph = 0, aph = 0;
      bool ok = true;
      const uint32_t full0 = tc::smem_u32(full), empty0 = tc::smem_u32(empty), acc_full0 = tc::smem_u32(acc_full), acc_empty0 = tc::smem_u32(acc_empty);
      const uint32_t ring_lo = (tc::smem_u32(ring) & 0x3FFFFu) >> 4, step = (uint32_t)g.stage_bytes >> 4, a_pl = (uint32_t)g.a_bytes >> 4, b_pl = (uint32_t)g.b_bytes >> 4;
      constexpr uint32_t A_LBO = 1u << 16, B_LBO = (B_MN ? 512u : 1u) << 16, B_STEP = B_MN ? 128u : 2u;  // a slice of 16 indices: 2048 or 32 bytes on
      for (int64_t u = unit; u < g.units && ok; u += units) {
        int in_chunk = 0;
        const int ku = (int)(u / g.per_k), kb1 = end_block(ku);
        for (int kb = first_block(ku); kb < kb1; ++kb) {
          if (in_chunk == 0) {
            if (!ht_wait<LIMIT>(acc_empty0 + 8 * as, aph ^ 1u, abort_flag)) { ok = false; break; }
            tc::tc_fence_after();
          }
          if (!ht_wait<LIMIT>(full0 + 8 * s, ph, abort_flag)) { ok = false; break; }
          tc::tc_fence_after();
          const uint32_t d = tmem_base + (uint32_t)as * acc_cols, a_hi = (ring_lo + s * step) | A_LBO, b_hi = (ring_lo + s * step + 2 * a_pl) | B_LBO;
          const bool last = in_chunk == kNsChunk - 1 || kb == kb1 - 1;
          if (!PAIR || one) {
            uint32_t more = in_chunk;
#pragma unroll
            for (int i = 0; i < kNsK / 16; ++i, more = 1) ht_mma<PAIR>(d, a_hi + a_pl + 2 * i, b_hi + B_STEP * i, g.idesc, more);
#pragma unroll
            for (int i = 0; i < kNsK / 16; ++i, more = 1) ht_mma<PAIR>(d, a_hi + 2 * i, b_hi + b_pl + B_STEP * i, g.idesc, more);
#pragma unroll
            for (int i = 0; i < kNsK / 16; ++i, more = 1) ht_mma<PAIR>(d, a_hi + 2 * i, b_hi + B_STEP * i, g.idesc, more);
            ht_commit<PAIR>(empty0 + 8 * s);
            if (last) ht_commit<PAIR>(acc_full0 + 8 * as);
          }
          if (++s == g.stages) { s = 0; ph ^= 1u; }
          ++in_chunk;
          if (last) {
            in_chunk = 0;
            if (++as == accs) { as = 0; aph ^= 1u; }
          }
        }
      }
      if (!ok) *abort_flag = 1;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kNsRegsDrain));
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t acc_empty_leader = PAIR ? tc::map_to_cta(tc::smem_u32(&acc_empty[0]), 0u) : 0u;
    int as = 0;
    uint32_t aph = 0;
    bool ok = true;
    for (int64_t u = unit; u < g.units; u += units) {
      int k, mt, nt;
      ns_tile<SYM, TM>(g, u, k, mt, nt);
      const int chunks = (end_block(k) - first_block(k) + kNsChunk - 1) / kNsChunk;
      const int64_t i = (int64_t)mt * TM + (int64_t)rank * 128 + quad * 32 + lane;
      const int64_t c_tile = (int64_t)nt * g.tile_n;
      const int nv = (int)min((int64_t)g.tile_n, g.n - c_tile);
      float l[4][32];  // this warp's blocks of 32 columns: half, half + 2, ...
      for (int ch = 0; ch < chunks && ok; ++ch) {
        // as a warp: what follows is for all of its lanes, or for none
        if (!__all_sync(~0u, tc::mbar_wait_limit(&acc_full[as], aph, abort_flag, LIMIT))) { ok = false; break; }
        tc::tc_fence_after();
        const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)as * acc_cols;
        if (ch == 0) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if ((2 * b + half) * 32 < nv) tc::tmem_ld32(taddr + (uint32_t)(2 * b + half) * 32, l[b]);
          tc::tmem_ld_wait();
#pragma unroll
          for (int b = 0; b < 4; ++b) tc::tmem_ld_arrived(l[b]);
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int c = (2 * b + half) * 32;
            if (c < nv) {
              float more[32];
              tc::tmem_ld32(taddr + (uint32_t)c, more);
              tc::tmem_ld_wait();
              tc::tmem_ld_arrived(more);
#pragma unroll
              for (int j = 0; j < 32; ++j) l[b][j] += more[j];
            }
          }
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) tc::mbar_arrive_cluster(acc_empty_leader + 8 * as);
          else tc::mbar_arrive(&acc_empty[as]);
        }
        if (++as == accs) { as = 0; aph ^= 1u; }
      }
      if (!ok) *abort_flag = 1;
      uint8_t* stage = stages + (warp - 4) * 4096;
      const int64_t i0 = i - lane;
      // one copy of the code for the four blocks: as straight code, run once a tile, it waited for its instructions (a block took 1.6 us, the result's 3.2)
#pragma unroll 1
      for (int b = 0; b < 4; ++b) {
        const int cb = (2 * b + half) * 32;
        if (cb >= nv || i0 >= g.m) break;
        const int64_t c = c_tile + cb;
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = (b < 2 ? b == 0 ? l[0][j] : l[1][j] : b == 2 ? l[2][j] : l[3][j]) * g.f;
        if (!ok) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = NAN;
        }
        if (!WHOLE) ns_stage_free(lane);
        if (EPI == NS_SQUARE && g.h != 0.f) ns_add_planes(v, g.h, g.other.p + (int64_t)k * 2 * g.other.plane, g.other.plane, g.other.ld, i0, g.m, c, stage, lane);
        if (WHOLE) {
          ns_store_final<T>(v, g, k, i0, c, reinterpret_cast<float*>(stage), lane);
        } else {
          if (EPI == NS_SQUARE && i0 == c) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += j == lane ? g.diagonal : 0.f;
          }
          ns_store_planes(v, &map_out, k, (int)i0, (int)c, stage, lane);
          // the transposed place belongs to no tile of the list: its column tile ends at or before its row tile's first column
          if (SYM && g.sym && (i0 / g.tile_n + 1) * g.tile_n <= c / TM * TM) ns_store_mirror(stage, g.out.p + (int64_t)k * 2 * g.out.plane, g.out.plane, g.out.ld, i0, c, g.n, lane);
        }
      }
    }
    if (!WHOLE && lane == 0) tc::bulk_wait_all<0>();
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // copies that may still be in flight land before shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) { }
    __syncthreads();
  }
  if (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after();
  if (warp == 1) {
    if (PAIR) tc::tmem_dealloc_pair(tmem_base, 512);
    else tc::tmem_dealloc(tmem_base, 512);
  }
}

// ------------------------------------------------------------------------------------------------ host side
// fp16 planes [2 K][rows][cols], columns contiguous: boxes of 64 columns x box_rows
inline bool ns_make_map(CUtensorMap* m, const NsPlanes& x, int64_t rows, int64_t cols, int32_t K, uint32_t box_rows, uint32_t box_cols = 64) {
  return ht_make_map<fp16>(m, x.p, (uint64_t)cols, (uint64_t)rows, (uint64_t)K * 2, x.ld, x.plane, box_rows, box_cols);
}

// The width of a tile: the one with the least work for the CTA (pair) that has most, of 256, 128 and, single, 64; a stage's loads weigh in as the columns
// that could be multiplied meanwhile.  A symmetric result takes half the tiles where that is less work, and all of them where idle SMs can have the rest: a tile
// whose transposed one is written as well ends 2 to 3 us later.
inline void ns_plan(NsGemm& g, int32_t K, bool sym, bool b_mn) {
  const bool pair = g.m > 128;
  const int tm = pair ? 256 : 128;
  const int64_t ctas = pair ? 74 : 148;
  g.m_tiles = (int)ceil_div(g.m, tm);
  double best = 1e300;
  for (int half = sym ? 1 : 0; half >= 0; --half)
    for (int n = 256; n >= (pair ? 128 : 64); n /= 2) {
      const int64_t n_tiles = ceil_div(g.n, n);
      int64_t per = 0;
      for (int i = 0; i < g.m_tiles; ++i) per += half ? n_tiles - std::min<int64_t>(n_tiles, (int64_t)i * tm / n) : n_tiles;
      const double cost = (double)ceil_div(per * K * g.splits, ctas) * (n + 48) + (half ? 1.0 : 0.0);
      if (cost < best) {
        best = cost;
        g.tile_n = n; g.n_tiles = (int)n_tiles; g.per_k = per; g.sym = half;
      }
    }
  g.units = g.per_k * K * g.splits;
  g.a_bytes = 128 * kNsK * 2;
  g.b_bytes = (pair ? g.tile_n / 2 : g.tile_n) * kNsK * 2;
  g.stage_bytes = 2 * (g.a_bytes + g.b_bytes);
  g.stages = std::min(kNsMaxStages, kNsRing / g.stage_bytes);
  g.idesc = tc::instr_desc(tm, g.tile_n, false, b_mn) & ~((1u << 7) | (1u << 10));  // operands f16
}

// Shares of a Gram matrix's inner indices: where its tiles leave most of the machine idle and a tile is long, so that a block of 64 indices, half a microsecond, is
// worth sharing (128 x 4096: one tile of 64 blocks, 35 us; shared by 16, and added up by another launch, 9).
inline int ns_splits(int32_t K, int64_t m, int64_t n) {
  const int64_t tiles = K * ceil_div(m, m > 128 ? 256 : 128) * ceil_div(m, 128), ctas = m > 128 ? 74 : 148, blocks = ceil_div(n, kNsK);
  const int64_t most = std::min(ctas / std::max<int64_t>(1, tiles), blocks / 4);
  if (most < 2 || blocks - blocks / most < 12) return 1;
  return (int)ceil_div(blocks, ceil_div(blocks, most));
}

// The shares' sums, in their order, as planes: 2^e times the Gram matrix.
__global__ void __launch_bounds__(256)
ns_join_kernel(const float* part, int splits, int64_t m, NsPlanes out, float f) {
  grid_dep_sync();
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, i = e / out.ld, at = (int64_t)blockIdx.y * 2 * out.plane + e;
  if (i >= m) return;
  const float* p = part + (int64_t)blockIdx.y * splits * m * out.ld + e;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int s = 0; s < splits; ++s) {
    const float4 w = *reinterpret_cast<const float4*>(p + (int64_t)s * m * out.ld);
    v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
  }
  union { uint2 q; __half2 h[2]; } a, b;
  ns_split2(v.x * f, v.y * f, a.h[0], b.h[0]);
  ns_split2(v.z * f, v.w * f, a.h[1], b.h[1]);
  *reinterpret_cast<uint2*>(out.p + at) = a.q;
  *reinterpret_cast<uint2*>(out.p + out.plane + at) = b.q;
}

template <typename T, int EPI>
inline cudaError_t ns_launch(const NsPlanes& A, const NsPlanes& B, NsGemm g, int32_t K, bool starved, cudaStream_t stream) {
  constexpr bool b_mn = EPI == NS_APPLY || EPI == NS_FINAL;
  if (EPI != NS_PART) { g.splits = 1; g.split_blocks = 0; }
  ns_plan(g, K, EPI == NS_GRAM || EPI == NS_SQUARE, b_mn);
  const bool pair = g.m > 128;
  CUtensorMap ma, mb, mo;
  if (!ns_make_map(&ma, A, g.m, g.inner, K, 128)) return cudaErrorInvalidValue;
  if (EPI == NS_FINAL || EPI == NS_PART) mo = ma;
  else if (!ns_make_map(&mo, g.out, g.m, g.n, K, 32, 32)) return cudaErrorInvalidValue;
  if (!(b_mn ? ns_make_map(&mb, B, g.inner, g.n, K, 64) : ns_make_map(&mb, B, g.n, g.inner, K, (uint32_t)(pair ? g.tile_n / 2 : g.tile_n)))) return cudaErrorInvalidValue;
  const void* kern = pair ? (const void*)ns_gemm_kernel<T, EPI, true, false> : (const void*)ns_gemm_kernel<T, EPI, false, false>;
  if constexpr (EPI != NS_FINAL || std::is_same<T, float>::value) {  // the self-test is of fp32 results
    if (starved) kern = pair ? (const void*)ns_gemm_kernel<T, EPI, true, true> : (const void*)ns_gemm_kernel<T, EPI, false, true>;
  }
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kNsSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(pair ? 2 * std::min<int64_t>(g.units, 74) : std::min<int64_t>(g.units, 148)));
  cfg.blockDim = dim3(kNsThreads); cfg.dynamicSmemBytes = kNsSmem; cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = pair ? 2 : 1;
  void* args[] = {&ma, &mb, &mo, &g};
  return cudaLaunchKernelExC(&cfg, kern, args);
}

// ------------------------------------------------------------------------------------------------ small matrices
// Up to kNsSmall rows, in one launch and in double: a cluster of blocks per matrix, a slice of the columns each.  The blocks add up their Gram matrices through distributed shared
// memory, and every one of them then takes the steps on m x m matrices alone: A <- P A P, Q <- P Q with P = a I + b A + c A^2, and multiplies its columns of G by Q.
// (In fp32 that would lose the small singular values, which A holds squared; in double they keep 1e-9 of the norm.)  The norm is the trace of A.
// 8 x 10 x 1024 fp32: 127 us in the products above, 17 launches; up to 64 rows (four times four results a thread) it was no faster than these.
constexpr int kNsSmall = 32;
template <int R> __host__ __device__ constexpr int ns_small_ld() { return 16 * R + 1; }
template <int R> __host__ __device__ constexpr int ns_small_smem() { return 8 * (5 * 16 * R * ns_small_ld<R>() + 16 * R * 65) + 64; }

// x y, and x z beside it (BOTH): matrices of m rows in M = 16 R, zeros behind them, rows LD apart; 16 x 16 threads, R x R results each, handed to `done`
template <int R, bool BOTH, class F>
__device__ __forceinline__ void ns_small_product(const double* x, const double* y, const double* z, int m, F&& done) {
  constexpr int LD = ns_small_ld<R>();
  const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
  double p[R][R] = {}, q[R][R] = {};
  for (int l0 = 0; l0 < m; l0 += 8)
#pragma unroll
    for (int l1 = 0; l1 < 8; ++l1) {
      const int l = l0 + l1;
      double f[R];
#pragma unroll
      for (int u = 0; u < R; ++u) f[u] = x[(ti + 16 * u) * LD + l];
#pragma unroll
      for (int v = 0; v < R; ++v) {
        const double yv = y[l * LD + tj + 16 * v], zv = BOTH ? z[l * LD + tj + 16 * v] : 0.0;
#pragma unroll
        for (int u = 0; u < R; ++u) {
          p[u][v] = fma(f[u], yv, p[u][v]);
          if (BOTH) q[u][v] = fma(f[u], zv, q[u][v]);
        }
      }
    }
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int v = 0; v < R; ++v) done(ti + 16 * u, tj + 16 * v, p[u][v], q[u][v]);
}

// 64 columns of the block's slice: on their way in registers, then in shared memory as double
template <typename T, int R>
struct NsSmallTile {
  static constexpr int M = 16 * R, E = M * 64 / 256;
  T f[E];
  __device__ __forceinline__ static int row(int e, bool along) { return along ? e >> 6 : e % M; }
  __device__ __forceinline__ static int col(int e, bool along) { return along ? e & 63 : e / M; }
  __device__ __forceinline__ void fetch(const T* g, int64_t si, int64_t sj, int m, int64_t c0, int64_t j1) {
    const bool along = sj <= si;  // read along the smaller stride
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const int e = threadIdx.x + u * 256, i = row(e, along), j = col(e, along);
      f[u] = i < m && c0 + j < j1 ? g[i * si + (c0 + j) * sj] : from_float<T>(0.f);
    }
  }
  __device__ __forceinline__ void put(double* tile, int64_t si, int64_t sj, double scale) const {
    const bool along = sj <= si;
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const int e = threadIdx.x + u * 256;
      tile[row(e, along) * 65 + col(e, along)] = (double)to_float(f[u]) * scale;
    }
  }
};

template <typename T, int R>
__global__ void __launch_bounds__(256)
ns_small_kernel(const T* g, int64_t sk, int64_t si, int64_t sj, int m, int64_t n, int64_t slice, int steps, double a, double b, double c, double scale, double eps, T* out, int64_t ok,
                int64_t oi, int64_t oj) {
  constexpr int LD = ns_small_ld<R>(), M = 16 * R;
  extern __shared__ double ns_small_words[];
  double *A = ns_small_words, *P = A + M * LD, *Q = P + M * LD, *W = Q + M * LD, *S = W + M * LD, *tile = S + M * LD;  // S: this block's sums, read by the cluster
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
  const int k = blockIdx.x / ranks, ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
  g += k * sk;
  out += k * ok;
  const int64_t j0 = min(n, (int64_t)rank * slice), j1 = min(n, j0 + slice);
  NsSmallTile<T, R> next;
  next.fetch(g, si, sj, m, j0, j1);
  double acc[R][R] = {};
  for (int64_t c0 = j0; c0 < j1; c0 += 64) {  // Gram matrix of the block's columns
    next.put(tile, si, sj, 1.0);
    __syncthreads();
    if (c0 + 64 < j1) next.fetch(g, si, sj, m, c0 + 64, j1);
#pragma unroll 8
    for (int j = 0; j < 64; ++j)
#pragma unroll
      for (int u = 0; u < R; ++u)
#pragma unroll
        for (int v = 0; v < R; ++v) acc[u][v] = fma(tile[(ti + 16 * u) * 65 + j], tile[(tj + 16 * v) * 65 + j], acc[u][v]);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int v = 0; v < R; ++v) S[(ti + 16 * u) * LD + tj + 16 * v] = acc[u][v];
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  next.fetch(g, si, sj, m, j0, j1);  // the first columns again, for the end
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int v = 0; v < R; ++v) {
      const int at = (ti + 16 * u) * LD + tj + 16 * v;
      const uint32_t here = tc::smem_u32(&S[at]);
      double d[8], sum = 0.0;
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r) {
        uint32_t there;
        d[r] = 0.0;
        if (r < ranks) {
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(r));
          asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(d[r]) : "r"(there) : "memory");
        }
      }
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r) sum += d[r];
      A[at] = sum;
      W[at] = 0.0;
    }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // waited for before S is written again: the steps' first product is the block's own
  __syncthreads();
  double trace = 0.0;
  for (int i = 0; i < m; ++i) trace += A[i * LD + i];
  const double inv = ns_inverse_of(trace, eps);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int v = 0; v < R; ++v) {
      const int i = ti + 16 * u, j = tj + 16 * v;
      A[i * LD + j] *= inv * inv;
      Q[i * LD + j] = i == j && i < m ? 1.0 : 0.0;
    }
  __syncthreads();
  for (int t = 0; t < steps; ++t) {
    const bool last = t + 1 == steps;
    ns_small_product<R, false>(A, A, nullptr, m, [&](int i, int j, double v, double) { P[i * LD + j] = fma(c, v, b * A[i * LD + j]) + (i == j && i < m ? a : 0.0); });
    __syncthreads();
    if (t == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // the cluster has read S
    if (last) {
      ns_small_product<R, false>(P, Q, nullptr, m, [&](int i, int j, double v, double) { S[i * LD + j] = v; });
    } else {
      ns_small_product<R, true>(P, A, Q, m, [&](int i, int j, double v, double q) {
        W[i * LD + j] = v;
        S[i * LD + j] = q;
      });
    }
    __syncthreads();
    double* s = Q; Q = S; S = s;
    if (last) break;
    ns_small_product<R, false>(W, P, nullptr, m, [&](int i, int j, double v, double) { A[i * LD + j] = v; });
    __syncthreads();
  }
  if (steps == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  const double f = inv * scale;
  for (int64_t c0 = j0; c0 < j1; c0 += 64) {  // the block's columns of Q G
    next.put(tile, si, sj, f);
    __syncthreads();
    if (c0 + 64 < j1) next.fetch(g, si, sj, m, c0 + 64, j1);
    const int w = (int)min((int64_t)64, j1 - c0);
    const bool along = oj <= oi;  // lanes along the smaller stride of the result
    const int pi = along ? ti : tj, pj = along ? tj : ti;
    double r[R][4] = {};
    for (int l0 = 0; l0 < m; l0 += 8)
#pragma unroll
      for (int l = l0; l < l0 + 8; ++l)
#pragma unroll
        for (int u = 0; u < R; ++u)
#pragma unroll
          for (int v = 0; v < 4; ++v) r[u][v] = fma(Q[(pi + 16 * u) * LD + l], tile[l * 65 + pj + 16 * v], r[u][v]);
#pragma unroll
    for (int u = 0; u < R; ++u)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (pi + 16 * u < m && pj + 16 * v < w) out[(pi + 16 * u) * oi + (c0 + pj + 16 * v) * oj] = from_float<T>((float)r[u][v]);
    __syncthreads();
  }
}

}  // namespace lsam
