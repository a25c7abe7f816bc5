// head_tcgen05.cuh -- scores of activations against a head on the 5th-generation tensor cores: the logits of a tile live in tensor
// memory only, and the warps that drain them keep the row statistics of head_ops.cuh instead of storing them.
//
// D(row, class) = sum_i h(row, i) w(class, i): rows on the M side, so a thread that drains tensor memory owns ONE row (its lane) and walks
// the classes of the tile in registers: no exchange between threads, the maximum, sum and entropy sum of a row stay in three registers over
// a run of tiles.  TMA stages 128B-swizzled tiles of 64 inner indices, one thread issues tcgen05.mma, eight warps drain (two per lane
// quadrant, alternate pairs of 32 columns); the accumulator is double-buffered so that a tile's statistics hide behind the next tile's products.
//   PAIR (more than 128 rows): two CTAs share 256 rows x tile_n classes (cta_group::2), each staging its own 128 rows of h and half the
//     classes; what bounds a CTA is the rate at which it takes in operands, 32 KB per 256 x 256 x 64 block instead of 48.
//   single CTA (up to 128 rows): the bytes of w bound it; only the rows that exist are loaded (the others' accumulator rows are never read).
// tile_n, a multiple of 32 (single CTAs: 16) up to 256, is the width that loads all SMs evenly.  The work list has the row tile fastest: the CTAs that run together
// read the same few tiles of w, so w crosses HBM once, whatever the number of row tiles.
// All waits are bounded as in gemm_tcgen05.cuh; a CTA that gives up leaves NaN statistics for its rows, and NaN for the logits of their labels.
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "head_score.cuh"
#include "tc_ptx.cuh"

namespace lsam {

// warp 0: TMA producer, warp 1: MMA issuer and tensor-memory owner, warps 2, 3: none; warps 4-11: draining (sixteen draining warps of half the
// logits each are slower: 2 x 353 x 135 x 32546 fp32 131 -> 171 us).  A draining thread holds the 128
// logits of its row's half tile, so the registers go to those two warpgroups: 56 + 2 x 216 a thread out of the 3 x 168 of the launch.
constexpr int kHtThreads = 384;
constexpr int kHtRegsIssue = 56, kHtRegsDrain = 216;
static_assert((kHtRegsIssue + 2 * kHtRegsDrain) * 128 <= 168 * kHtThreads, "setmaxnreg draws on the registers of the launch");
constexpr int kHtRows = 128, kHtMaxN = 256, kHtK = 64;
constexpr int kHtBlocks = kHtMaxN / 64;  // blocks of 32 classes a draining warp owns
// The tensor core cuts off, not rounds, what lies below the accumulator's last place, at every step of 16 inner indices: a sum of 4096 terms
// came out 2e-6 short.  So a tile's products are summed in chunks of kHtChunk blocks of 64, each in an accumulator of its own, and the chunks
// are added in registers.
constexpr int kHtChunk = 12;
constexpr int kHtMaxStages = 12, kHtRing = 216 * 1024;  // bytes of the ring
constexpr int kHtBiasBytes = 8 * kHtBlocks * 32 * 4;  // a tile's bias, per draining warp
constexpr int kHtSmem = kHtRing + 1024 + 512 + kHtBiasBytes;

struct HeadTile {
  int tile_n, run;     // classes of a tile, consecutive tiles of a unit of work
  int n_tiles, m_tiles, runs;
  int a_rows;          // rows of h a load brings in (a multiple of 8, at most 128)
  int stages, stage_bytes, a_bytes;  // the ring: [h tile][w tile] per stage, each on a 1024-byte boundary
  int w_shared;        // one head for all workers
  int pairs;           // 1, or 6: fp32 operands as three bf16 planes, plane p of worker k at index k + p K of the maps
  uint32_t idesc;
  int K;
  int64_t units;       // K * runs * m_tiles
};

// What the issuing warps do per block of 64 inner indices has to stay below the 512 clocks of a 256-wide tile's products.  Barriers and operands are
// addressed by 32-bit shared-memory addresses, and of a matrix descriptor (tc::smem_desc with leading offset 16, stride offset 1024) only the low word
// changes.  The one thread that issues is chosen by elect.sync: tcgen05 instructions take uniform registers, and under a test of the lane number the
// compiler, which cannot know that one thread is active, guards every one of them (475 clocks a block beside the products; 4096 x 4096 x 32768:
// 937 -> 784 us).  A pair's warps walk their loops whole and elect at the instruction (707 us); single CTAs elect once (4 rows: 59 -> 54 us).
__device__ inline bool ht_elect() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
template <uint32_t LIMIT>
__device__ inline bool ht_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < LIMIT; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
    if ((i & 1023u) == 1023u && *abort_flag) return false;
  }
  return false;
}
constexpr uint32_t kHtDescHi = 64u | (1u << 14) | (2u << 29);
__device__ inline uint32_t ht_desc_lo(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | (1u << 16); }
template <bool PAIR>
__device__ inline void ht_mma(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kHtDescHi) : "memory");
  else
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kHtDescHi) : "memory");
}
template <bool PAIR>
__device__ inline void ht_commit(uint32_t bar) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <bool PAIR>
__device__ inline void ht_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  if (PAIR)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}

// The statistics of 32 logits of a row: classes c0 .. c0 + 31, of which `have` exist.  bias: their 32 values in shared memory, or null.  *at_label receives the label's logit.
__device__ __forceinline__ void ht_block_stats(float (&l)[32], RowStat& st, int64_t c0, int have, const float* bias, int32_t y, float* at_label) {
  if (bias != nullptr) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float4 v = reinterpret_cast<const float4*>(bias)[q];
      l[4 * q] += v.x; l[4 * q + 1] += v.y; l[4 * q + 2] += v.z; l[4 * q + 3] += v.w;
    }
  }
  if (have < 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j) l[j] = j < have ? l[j] : kMasked;
  }
  const int64_t at = (int64_t)y - c0;
  if (at >= 0 && at < 32 && at < have) {
    float lab = 0.f;
    // a select per element in PTX: written as an index, or as anything the compiler can turn into one, it puts the array into local memory
#pragma unroll
    for (int j = 0; j < 32; ++j)
      asm("{\n.reg .pred p;\nsetp.eq.s32 p, %1, %2;\n@p mov.f32 %0, %3;\n}\n" : "+f"(lab) : "r"((int)at), "r"(j), "f"(l[j]));
    *at_label = lab;
  }
  float mx[4] = {st.m, st.m, st.m, st.m};  // four chains
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    l[j] = max_nan(l[j], kMasked);
    mx[j & 3] = fmaxf(mx[j & 3], l[j]);
  }
  stat_add_all(st, l, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
}

// fp32 operands arrive as three bf16 planes each (head_copy_kernel) and six products of planes are accumulated, as in the fp32 models' GEMMs.
// grid: CTAs (pairs: clusters of 2), each walking units u, u + grid, ...; unit = (run of class tiles, row tile) of a worker, row tile fastest
// STARVED (self-test): no copy is ever issued and the waits are short, so all of them run out with nothing in flight.
template <bool PAIR, bool STARVED>
__global__ void __launch_bounds__(kHtThreads, 1)
head_tcgen05_kernel(const __grid_constant__ CUtensorMap map_h, const __grid_constant__ CUtensorMap map_w, HeadArgs a, HeadTile q) {
  constexpr uint32_t LIMIT = STARVED ? 1u << 13 : tc::kSpinLimit;
  const int STAGES = q.stages, A_BYTES = q.a_bytes, STAGE = q.stage_bytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + kHtRing);  // [stages]
  uint64_t* empty = full + kHtMaxStages;
  uint64_t* acc_full = empty + kHtMaxStages;  // [2]
  uint64_t* acc_empty = acc_full + 2;    // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kHtMaxStages + 4) * 8 + 8 <= 512 && kHtSmem <= 227 * 1024, "barrier area");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? tc::cluster_ctarank() : 0u;
  const bool leader = rank == 0u;
  const int64_t unit = PAIR ? blockIdx.x / 2 : blockIdx.x, units = PAIR ? gridDim.x / 2 : gridDim.x;
  const int k_blocks = (int)((a.inner + kHtK - 1) / kHtK), k_total = q.pairs * k_blocks, chunks = (k_total + kHtChunk - 1) / kHtChunk;
  const int b_rows = PAIR ? q.tile_n / 2 : q.tile_n;  // classes staged by this CTA
  const uint32_t stage_tx = (uint32_t)(q.a_rows + b_rows) * kHtK * 2;

  grid_dep_launch();
  if (threadIdx.x == 0) {
    tc::prefetch_tensormap(&map_h);
    tc::prefetch_tensormap(&map_w);
    for (int s = 0; s < STAGES; ++s) { tc::mbar_init(&full[s], 1); tc::mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { tc::mbar_init(&acc_full[s], 1); tc::mbar_init(&acc_empty[s], PAIR ? 16 : 8); }
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
  const uint32_t tmem_base = *tmem_slot;  // 512 columns: the whole tensor memory, so 0 in both CTAs of a pair

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHtRegsIssue));
    const bool one = ht_elect();
    if (!STARVED && warp == 0 && (PAIR || one)) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      const uint32_t ring0 = tc::smem_u32(ring), full0 = tc::smem_u32(full), empty0 = tc::smem_u32(empty);
      // both CTAs' loads of a stage complete on the leader's barrier, which the leader arms with the bytes of both
      const uint32_t bar0 = PAIR ? tc::map_to_cta(full0, 0u) : full0, tx = PAIR ? 2 * stage_tx : stage_tx;
      for (int64_t u = unit; u < q.units && ok; u += units) {
        const int mt = (int)(u % q.m_tiles), rn = (int)((u / q.m_tiles) % q.runs), k = (int)(u / ((int64_t)q.m_tiles * q.runs));
        const int r0 = (mt * (PAIR ? 2 : 1) + (int)rank) * kHtRows, kw = q.w_shared ? 0 : k;
        const int nt_end = min(q.n_tiles, (rn + 1) * q.run);
        for (int nt = rn * q.run; nt < nt_end && ok; ++nt) {
          const int c0 = nt * q.tile_n + (int)rank * b_rows;
          for (int pp = 0; pp < q.pairs && ok; ++pp) {
            // plane pairs (0,2) (1,1) (2,0) (0,1) (1,0) (0,0): the small products first, the rest below 2^-24 of |h| |w| left out
            const int pa = q.pairs == 1 ? 0 : pp < 3 ? pp : pp < 5 ? pp - 3 : 0, pb = q.pairs == 1 ? 0 : pp < 3 ? 2 - pp : pp < 5 ? 4 - pp : 0;
            const int zh = k + pa * q.K, zw = q.w_shared ? pb : kw + pb * q.K;
            for (int kb = 0; kb < k_blocks; ++kb) {
              if (!ht_wait<LIMIT>(empty0 + 8 * s, ph ^ 1u, abort_flag)) { ok = false; break; }
              const uint32_t dst = ring0 + s * STAGE;
              if (!PAIR || one) {
                if (!PAIR || leader) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full0 + 8 * s), "r"(tx) : "memory");
                ht_load<PAIR>(dst, &map_h, kb * kHtK, r0, zh, bar0 + 8 * s);
                ht_load<PAIR>(dst + A_BYTES, &map_w, kb * kHtK, c0, zw, bar0 + 8 * s);
              }
              if (++s == STAGES) { s = 0; ph ^= 1u; }
            }
          }
        }
      }
      if (!ok) *abort_flag = 1;
    }
    if (warp == 1 && leader && (PAIR || one)) {
      int s = 0, as = 0;
      uint32_t ph = 0, aph = 0;
      bool ok = true;
      const uint32_t full0 = tc::smem_u32(full), empty0 = tc::smem_u32(empty), acc_full0 = tc::smem_u32(acc_full), acc_empty0 = tc::smem_u32(acc_empty);
      const uint32_t lo0 = ht_desc_lo(tc::smem_u32(ring)), step = (uint32_t)STAGE >> 4, b_off = (uint32_t)A_BYTES >> 4;
      for (int64_t u = unit; u < q.units && ok; u += units) {
        const int rn = (int)((u / q.m_tiles) % q.runs), nt_end = min(q.n_tiles, (rn + 1) * q.run);
        for (int nt = rn * q.run; nt < nt_end && ok; ++nt) {
          int in_chunk = 0;
          for (int kb = 0; kb < k_total; ++kb) {
            if (in_chunk == 0) {
              if (!ht_wait<LIMIT>(acc_empty0 + 8 * as, aph ^ 1u, abort_flag)) { ok = false; break; }
              tc::tc_fence_after();
            }
            if (!ht_wait<LIMIT>(full0 + 8 * s, ph, abort_flag)) { ok = false; break; }
            const uint32_t d = tmem_base + (uint32_t)as * kHtMaxN, a_lo = lo0 + s * step, b_lo = a_lo + b_off;
            const bool last = in_chunk == kHtChunk - 1 || kb == k_total - 1;
            if (!PAIR || one) {
#pragma unroll
              for (int k = 0; k < kHtK / 16; ++k) ht_mma<PAIR>(d, a_lo + 2 * k, b_lo + 2 * k, q.idesc, in_chunk + k);  // 16 indices are 32 bytes along the row
              ht_commit<PAIR>(empty0 + 8 * s);
              if (last) ht_commit<PAIR>(acc_full0 + 8 * as);
            }
            if (++s == STAGES) { s = 0; ph ^= 1u; }
            ++in_chunk;
            if (last) {
              in_chunk = 0;
              if (++as == 2) { as = 0; aph ^= 1u; }
            }
          }
        }
      }
      if (!ok) *abort_flag = 1;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kHtRegsDrain));
    const int quad = warp & 3, half = (warp - 4) >> 2;
    float* my_bias = reinterpret_cast<float*>(ring + kHtRing + 512) + (warp - 4) * (kHtBlocks * 32);
    const uint32_t acc_empty_leader[2] = {PAIR ? tc::map_to_cta(tc::smem_u32(&acc_empty[0]), 0u) : 0u, PAIR ? tc::map_to_cta(tc::smem_u32(&acc_empty[1]), 0u) : 0u};
    int as = 0;
    uint32_t aph = 0;
    bool ok = true;
    for (int64_t u = unit; u < q.units; u += units) {  // every unit, also after giving up: its statistics are then NaN
      const int mt = (int)(u % q.m_tiles), rn = (int)((u / q.m_tiles) % q.runs), k = (int)(u / ((int64_t)q.m_tiles * q.runs));
      const int64_t r = (int64_t)(mt * (PAIR ? 2 : 1) + (int)rank) * kHtRows + quad * 32 + lane;
      const bool live = r < a.rows;
      const int64_t i = (int64_t)k * a.rows + r;
      const int32_t y = (live && a.labels) ? a.labels[i] : -1;
      const float* bias = a.bias ? a.bias + k * a.bk : nullptr;
      RowStat st = stat_empty();
      const int nt_end = min(q.n_tiles, (rn + 1) * q.run);
      for (int nt = rn * q.run; nt < nt_end && ok; ++nt) {
        const int64_t c_tile = (int64_t)nt * q.tile_n;
        const int nv = (int)min((int64_t)q.tile_n, a.classes - c_tile);  // classes that exist
        float l[kHtBlocks][32];  // this warp's blocks of 32 classes: half, half + 2, ...
        // The bias of these classes, a value a lane, is asked for while the products run and read by all lanes from shared memory, four at a time: as 32
        // loads of the same address by all lanes it cost as much as the statistics (2048 x 512 x 32768 with bias: 96 us, now 74).
        float bv[kHtBlocks];
#pragma unroll
        for (int b = 0; b < kHtBlocks; ++b) {
          const int c = (2 * b + half) * 32 + lane;
          bv[b] = bias && c < nv ? __ldg(bias + c_tile + c) : 0.f;
        }
        for (int ch = 0; ch < chunks && ok; ++ch) {
          if (!tc::mbar_wait_limit(&acc_full[as], aph, abort_flag, LIMIT)) { ok = false; break; }
          tc::tc_fence_after();
          const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)as * kHtMaxN;
          if (ch == 0) {  // all of them in flight at once
#pragma unroll
            for (int b = 0; b < kHtBlocks; ++b)
              if ((2 * b + half) * 32 < nv) tc::tmem_ld32(taddr + (uint32_t)(2 * b + half) * 32, l[b]);
            tc::tmem_ld_wait();
#pragma unroll
            for (int b = 0; b < kHtBlocks; ++b) tc::tmem_ld_arrived(l[b]);
          } else {
#pragma unroll
            for (int b = 0; b < kHtBlocks; ++b) {
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
            if (PAIR) tc::mbar_arrive_cluster(acc_empty_leader[as]);
            else tc::mbar_arrive(&acc_empty[as]);
          }
          if (++as == 2) { as = 0; aph ^= 1u; }
        }
        if (!ok) break;
        if (bias) {
          __syncwarp();  // the last tile's have been read
#pragma unroll
          for (int b = 0; b < kHtBlocks; ++b) my_bias[b * 32 + lane] = bv[b];
          __syncwarp();
        }
#pragma unroll
        for (int b = 0; b < kHtBlocks; ++b) {
          const int c = (2 * b + half) * 32;
          if (c < nv) ht_block_stats(l[b], st, c_tile + c, nv - c, bias ? my_bias + b * 32 : nullptr, y, a.at_label + i);
        }
      }
      if (!ok) {
        *abort_flag = 1;
        st = {0.f, NAN, NAN};
        // nobody may have written the logit of a label in these classes: what is there is the workspace's, and must not pass for a mask
        if (live && y >= (int64_t)rn * q.run * q.tile_n && y < (int64_t)nt_end * q.tile_n) a.at_label[i] = NAN;
      }
      if (live) a.part[(int64_t)(rn * 2 + half) * a.total + i] = st;
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // copies that may still be in flight land before shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) { }
    __syncthreads();
  }
  // neither CTA of a pair leaves while the other can still read its shared memory, write its barriers or fill its tensor memory
  if (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after();
  if (warp == 1) {
    if (PAIR) tc::tmem_dealloc_pair(tmem_base, 512);
    else tc::tmem_dealloc(tmem_base, 512);
  }
}

// ------------------------------------------------------------------------------------------------ host side
// The width of a tile and the run of tiles that load the machine most evenly: the CTAs (pairs) work through ceil(units / CTAs) rounds of `run`
// tiles.  A pair's tile costs its width plus the share of h it takes in (32 classes' worth); a single CTA's, whose bytes of w count, its width, plus a
// little per tile and the last tile's statistics, which nothing hides.  Longer runs leave fewer partial statistics.  The first of equals in the order of
// falling widths, then runs.  What cannot be cheaper than one guess per width is passed over: 0.3 to 1 us on the host (the whole search: 0.3 to 4.5).
inline HeadTile ht_plan(int32_t K, int64_t rows, int64_t classes) {
  HeadTile q{};
  const bool pair = rows > kHtRows;
  const int64_t ctas = pair ? 74 : 148;
  q.m_tiles = (int)ceil_div(rows, pair ? 2 * kHtRows : kHtRows);
  const int64_t km = (int64_t)K * q.m_tiles;
  const int grain = pair ? 32 : 16;  // the multiple of 16 that tcgen05.mma wants, in each CTA of a pair
  // `tiles`: those of the CTA that has most
  const auto price = [&](double tiles, int n, int64_t run) { return (pair ? tiles * (n + 32) : tiles * (n + 8) + 0.25 * n) * (1.0 + 0.02 / run); };
  const auto cost = [&](int n, int64_t n_tiles, int64_t run) { return price((double)ceil_div(km * ceil_div(n_tiles, run), ctas) * run, n, run); };
  double best = 1e300;
  for (int n = kHtMaxN; n >= 32; n -= grain) {
    const int64_t n_tiles = ceil_div(classes, (int64_t)n);
    best = std::min(best, cost(n, n_tiles, std::min(std::min<int64_t>(n_tiles, 32), ceil_div(km * n_tiles, ctas))));
  }
  best *= 1.0 + 1e-9;  // the guess itself is to be found again
  for (int n = kHtMaxN; n >= 32; n -= grain) {
    const int64_t n_tiles = ceil_div(classes, (int64_t)n), longest = std::min<int64_t>(n_tiles, 32);
    const double even = std::max(1.0, (double)(km * n_tiles) / ctas) * (1.0 - 1e-9);  // no CTA has fewer if all have alike
    if (price(even, n, longest) >= best) continue;
    const double most = (best - (pair ? 0.0 : 0.25 * n)) / (pair ? n + 32 : n + 8);  // a cheaper plan has fewer tiles a CTA, so no longer run
    for (int64_t run = std::min(longest, (int64_t)most); run >= 1 && price(even, n, run) < best; --run) {
      const double c = cost(n, n_tiles, run);
      if (c < best) {
        best = c;
        q.tile_n = n; q.run = (int)run; q.n_tiles = (int)n_tiles; q.runs = (int)ceil_div(n_tiles, run);
      }
    }
  }
  q.units = (int64_t)K * q.m_tiles * q.runs;
  q.a_rows = pair ? kHtRows : (int)round_up(rows, 8);
  // few rows: the h tile is as small as they are, and the ring as deep as it can be (the rows of the tile that are not there are whatever lies
  // behind it in the ring, which leaves the accumulators of the rows that are alone)
  q.a_bytes = (int)round_up(q.a_rows * kHtK * 2, 1024);
  q.stage_bytes = q.a_bytes + (pair ? q.tile_n / 2 : q.tile_n) * kHtK * 2;
  q.stages = std::min(kHtMaxStages, kHtRing / q.stage_bytes);
  while ((q.stages - 1) * q.stage_bytes + kHtRows * kHtK * 2 > kHtRing) --q.stages;  // 128 rows' worth behind the last stage's start
  return q;
}

// 16-bit tensor [Z][rows][inner], inner contiguous; boxes of 64 inner indices x box_rows
template <typename T>
inline bool ht_make_map(CUtensorMap* m, const T* base, uint64_t inner, uint64_t rows, uint64_t Z, int64_t row_stride, int64_t z_stride, uint32_t box_rows) {
  PFN_encodeTiled enc = tc_encode_fn();
  if (!enc) return false;
  // the stride of a dimension of one element is never used, but has to be a legal one
  const uint64_t rs = rows > 1 ? (uint64_t)row_stride * 2 : (uint64_t)round_up((int64_t)inner * 2, 16);
  const uint64_t zs = Z > 1 ? (uint64_t)z_stride * 2 : rs;
  if ((reinterpret_cast<uintptr_t>(base) & 15) || rs % 16 || zs % 16 || rs == 0 || zs == 0 || rs >= ((uint64_t)1 << 40) || zs >= ((uint64_t)1 << 40)) return false;
  cuuint64_t dims[3] = {inner, rows, Z};
  cuuint64_t strides[2] = {rs, zs};
  cuuint32_t box[3] = {(cuuint32_t)kHtK, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(m, std::is_same<T, bf16>::value ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<T*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// False (nothing launched): the operands' addresses or strides are not what TMA takes.  *e: the launch's error.
template <typename T>
inline bool ht_launch(const T* h, const T* w, HeadArgs a, int32_t K, HeadTile q, int planes, bool shared, bool starved, cudaStream_t stream, cudaError_t* e) {
  const bool pair = a.rows > kHtRows;
  CUtensorMap mh, mw;
  q.w_shared = shared;
  q.K = K;
  q.pairs = planes == 3 ? 6 : 1;
  if (!ht_make_map(&mh, h, a.inner, a.rows, (uint64_t)K * planes, a.hr, a.hk, (uint32_t)q.a_rows)) return false;
  if (!ht_make_map(&mw, w, a.inner, a.classes, (uint64_t)(q.w_shared ? 1 : K) * planes, a.wr, a.wk, (uint32_t)(pair ? q.tile_n / 2 : q.tile_n))) return false;
  q.idesc = tc::instr_desc(pair ? 256 : 128, q.tile_n, false, false);
  if (!std::is_same<T, bf16>::value) q.idesc &= ~((1u << 7) | (1u << 10));  // operands f16 instead of bf16
  a.parts = 2 * q.runs;
  const void* kern = starved ? (pair ? (const void*)head_tcgen05_kernel<true, true> : (const void*)head_tcgen05_kernel<false, true>)
                             : (pair ? (const void*)head_tcgen05_kernel<true, false> : (const void*)head_tcgen05_kernel<false, false>);
  const int smem = kHtSmem;
  if ((*e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return true;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(pair ? 2 * std::min<int64_t>(q.units, 74) : std::min<int64_t>(q.units, 148)));
  cfg.blockDim = dim3(kHtThreads); cfg.dynamicSmemBytes = smem; cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = pair ? 1 : 0;
  void* args[] = {&mh, &mw, &a, &q};
  *e = cudaLaunchKernelExC(&cfg, kern, args);
  return true;
}

}  // namespace lsam
