// layer_api.cu -- host side of the operators for the layers and the update of a model of the caller's own (include/lsam.h, last section): argument
// checks and launches.  Nothing here allocates, synchronises or keeps state between calls.
#include "lsam.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "embed.cuh"
#include "op_check.cuh"
#include "orthogonalize.cuh"
#include "residual_norm.cuh"

using namespace lsam;

namespace {

constexpr int64_t kMaxWide = (int64_t)1 << 30;

// A launch behind a kernel of the same call: its blocks become resident while that one drains, and wait for it there.
template <typename... P, typename... A>
cudaError_t launch_behind(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}

// Rows [n0, n1] of a tensor that start on 16-byte boundaries.
bool rows_aligned(const void* p, size_t es, int64_t n0, int64_t s0, int64_t n1, int64_t s1) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (n0 == 1 || s0 * (int64_t)es % 16 == 0) && (n1 == 1 || s1 * (int64_t)es % 16 == 0);
}

}  // namespace

extern "C" int lsam_embed(const void* d_table, int32_t dtype, int32_t K, int64_t rows, int64_t vocab, int64_t n, int64_t table_stride_k, int64_t table_stride_row,
                          const int32_t* d_tokens, float scale, void* d_out, int64_t out_stride_k, int64_t out_stride_row, void* cuda_stream, char* h_err, size_t h_err_len) {
  const Err err("lsam_embed", h_err, h_err_len);
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (K < 0 || rows < 0 || n < 0 || vocab < 1 || vocab > kMaxWide || n > kMaxWide) return err.fail(LSAM_ERR_INVALID, "need K, rows, n >= 0, 1 <= vocab <= 2^30, n <= 2^30");
  if (K == 0 || rows == 0 || n == 0) return LSAM_OK;
  if (rows > kMaxIndex / K) return err.fail(LSAM_ERR_INVALID, "K * rows must be below 2^31");
  if (!strides_ok(K, table_stride_k, vocab, table_stride_row, n, 1) || !strides_ok(K, out_stride_k, rows, out_stride_row, n, 1))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or a tensor is too large");
  if (!disjoint(K, out_stride_k, rows, out_stride_row, n, 1)) return err.fail(LSAM_ERR_INVALID, "elements of the output share an address or interleave");
  const size_t es = dtype_size(dtype);
  PtrCheck pc;
  pc.need(d_table, es); pc.need(d_out, es); pc.need(d_tokens, 4);
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  const EmbedArgs a{d_tokens, rows, n, vocab, table_stride_k, table_stride_row, out_stride_k, out_stride_row, scale, FastDiv((uint32_t)rows), 0};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool vec = rows_aligned(d_table, es, K, table_stride_k, vocab, table_stride_row) && rows_aligned(d_out, es, K, out_stride_k, rows, out_stride_row);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const uint64_t per_row = vec ? (uint64_t)ceil_div(n, vec_n<T>()) : (uint64_t)n, units = per_row * K * rows, blocks = (units + 256 * kEmbedUnroll - 1) / (256 * kEmbedUnroll);
    if (blocks > (uint64_t)kMaxIndex) { e = cudaErrorInvalidConfiguration; return; }
    const auto go = [&](auto kern) {
      kern<<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const T*>(d_table), static_cast<T*>(d_out), a, FastDiv((uint32_t)per_row), units);
      return cudaPeekAtLastError();
    };
    e = vec ? go(embed_kernel<T, true>) : go(embed_kernel<T, false>);
  });
  return err.done(e);
}

namespace {

// Where a gradient call's threads are and what its workspace holds.  A thread takes 16 bytes of a row (E elements); `lanes` of them walk a tile.
// Tiles are as long as leaves 2048 threads an SM (fewer partial sums), at least 8 rows.
struct EmbedPlan {
  int64_t lists, N, chunks, tiles, width;
  int lanes, tile, E;
  SortPlan sort;
  size_t b, part, open, total;
};
bool embed_grad_sizes_ok(int32_t K, int64_t rows, int64_t vocab, int64_t n) {
  return K >= 1 && K <= 65535 && rows >= 1 && n >= 1 && vocab >= 1 && vocab <= kMaxWide && n <= kMaxWide && rows <= kMaxIndex / K && vocab <= kMaxIndex / K;
}
EmbedPlan embed_plan(int32_t dtype, int32_t K, int64_t rows, int64_t vocab, int64_t n, bool shared) {
  EmbedPlan p{};
  p.lists = shared ? 1 : K;
  p.N = shared ? K * rows : rows;
  p.E = dtype == LSAM_FP32 ? 4 : 8;  // the element-wise form takes 4 as well: the width below covers both
  const int64_t per_row = ceil_div(n, p.E);
  p.lanes = 1;
  while (p.lanes < 256 && p.lanes < per_row) p.lanes *= 2;
  p.chunks = ceil_div(per_row, p.lanes);
  p.tile = 64;
  while (p.tile > 8 && p.lists * ceil_div(p.N, p.tile) * p.chunks * p.lanes < 148 * 2048) p.tile /= 2;
  p.tiles = ceil_div(p.N, p.tile);
  p.width = p.chunks * p.lanes * p.E;
  p.sort = sort_plan(p.N, vocab);
  p.b = (size_t)round_up(8 * p.lists * p.N, 256);
  p.part = 2 * p.b;
  p.open = p.part + (size_t)round_up(8 * p.lists * p.tiles * p.width, 256);
  p.total = p.open + (size_t)round_up(4 * (1 + p.lists * p.tiles), 256);
  return p;
}

// The sort and, unless rows of other tokens are to stay as they are, the zeros: ranges of tokens that give every SM eight blocks of
// them, three at a time, if there are enough (512 ranges of 64 left a second wave of 29: 80 us instead of 62); three where each has many tokens to look through.
template <typename TG>
cudaError_t launch_sort(const EmbedArgs& a, TG* grad, const EmbedLists& L, const EmbedPlan& p, bool accumulate, cudaStream_t stream) {
  const int cluster = p.N > 0 ? p.sort.cluster : 1;
  const int64_t sort_blocks = p.N > 0 ? p.lists * cluster : 0;
  EmbedZero z{grad, a.n, a.vocab, a.tk, a.tr, 1, 1, 0};
  if (!accumulate) {
    z.range = (int32_t)std::min<int64_t>(kZeroRange, std::max<int64_t>(8, ceil_div(a.vocab * p.lists, (p.N <= 65536 ? 8 : 3) * 148)));
    z.per_list = (uint32_t)ceil_div(a.vocab, (int64_t)z.range);
    z.blocks = z.per_list * (uint32_t)p.lists;
  }
  const int64_t blocks = round_up(sort_blocks + z.blocks, cluster);
  if (blocks == 0) return cudaSuccess;
  const auto kern = embed_sort_kernel<TG>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sort_smem(kSortBits));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(kSortThreads); cfg.dynamicSmemBytes = (size_t)std::max(p.N > 0 ? sort_smem(p.sort.bits) : 0, z.range / 8 + 4);
  cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, a.tokens, a.vocab, L, p.sort.bits, p.sort.passes, p.sort.per, (uint32_t)sort_blocks, z);
}

template <typename T, typename TG>
cudaError_t launch_embed_grad(const T* dout, TG* grad, const EmbedArgs& a, const EmbedPlan& p, const EmbedLists& L, bool vec, bool vec_out, bool accumulate, cudaStream_t stream) {
  const int64_t chunks = ceil_div(a.n, (vec ? vec_n<T>() : 4) * (int64_t)p.lanes), quads = ceil_div(a.n, 4);
  int lanes = 1;
  while (lanes < 256 && lanes < quads) lanes *= 2;
  if (p.lists * p.tiles * std::max(chunks, ceil_div(quads, lanes)) > kMaxIndex) return cudaErrorInvalidConfiguration;
  cudaError_t e = launch_sort<TG>(a, grad, L, p, accumulate, stream);
  if (e != cudaSuccess || p.N == 0) return e;
  const auto grid = [&](int lanes, int64_t chunks) {
    EmbedGrid g;
    g.lanes = lanes;
    g.units = (uint32_t)(p.lists * p.tiles * chunks);
    g.by_chunks = FastDiv((uint32_t)chunks);
    g.by_tiles = FastDiv((uint32_t)p.tiles);
    g.vec_out = vec_out;
    g.accumulate = accumulate;
    return g;
  };
  const EmbedGrid g = grid(p.lanes, chunks), h = grid(lanes, ceil_div(quads, lanes));
  const dim3 blocks((unsigned)ceil_div(g.units, 256 / g.lanes));
  e = vec ? launch_behind(embed_sum_kernel<T, TG, true>, blocks, dim3(256), 0, stream, dout, grad, a, L, g) : launch_behind(embed_sum_kernel<T, TG, false>, blocks, dim3(256), 0, stream, dout, grad, a, L, g);
  if (e == cudaSuccess && p.tiles > 1) e = launch_behind(embed_join_kernel<TG>, dim3((unsigned)std::min<int64_t>(ceil_div(h.units, 256 / h.lanes), 4 * 148)), dim3(256), 0, stream, grad, a, L, h);
  return e;
}

}  // namespace

extern "C" size_t lsam_embed_grad_workspace_bytes(int32_t dtype, int32_t K, int64_t rows, int64_t vocab, int64_t n, int32_t shared) {
  if (!dtype_ok(dtype) || !embed_grad_sizes_ok(K, rows, vocab, n)) return 0;
  return embed_plan(dtype, K, rows, vocab, n, shared != 0 || K == 1).total;
}

extern "C" int lsam_embed_grad(const void* d_dout, int32_t dtype, int32_t K, int64_t rows, int64_t vocab, int64_t n, int64_t dout_stride_k, int64_t dout_stride_row,
                               const int32_t* d_tokens, float scale, void* d_grad, int32_t grad_dtype, int64_t grad_stride_k, int64_t grad_stride_row, int32_t accumulate,
                               void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* h_err, size_t h_err_len) {
  const Err err("lsam_embed_grad", h_err, h_err_len);
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (grad_dtype != dtype && grad_dtype != LSAM_FP32) return err.fail(LSAM_ERR_INVALID, "grad_dtype must be dtype or LSAM_FP32");
  if (K < 0 || rows < 0 || n < 0 || vocab < 1 || vocab > kMaxWide || n > kMaxWide) return err.fail(LSAM_ERR_INVALID, "need K, rows, n >= 0, 1 <= vocab <= 2^30, n <= 2^30");
  if (n == 0) return LSAM_OK;
  if (K == 0) {  // no workers: nothing but the zeros of a gradient that they would share
    if (grad_stride_k != 0 || accumulate) return LSAM_OK;
    K = 1;
    rows = 0;
  }
  const bool shared = grad_stride_k == 0 || K == 1;
  const int64_t lists = shared ? 1 : K;
  if (K > 65535 || rows > kMaxIndex / K || vocab > kMaxIndex / K) return err.fail(LSAM_ERR_INVALID, "need K <= 65535, K * rows and K * vocab below 2^31");
  if (!strides_ok(K, dout_stride_k, rows > 0 ? rows : 1, dout_stride_row, n, 1) || !strides_ok(lists, grad_stride_k, vocab, grad_stride_row, n, 1))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or a tensor is too large");
  if (!disjoint(lists, grad_stride_k, vocab, grad_stride_row, n, 1)) return err.fail(LSAM_ERR_INVALID, "elements of the gradient share an address or interleave");
  const size_t es = dtype_size(dtype), gs = dtype_size(grad_dtype);
  PtrCheck pc;
  pc.need(d_grad, gs);
  if (rows == 0 && accumulate) return LSAM_OK;
  const EmbedPlan p = embed_plan(dtype, K, rows, vocab, n, shared);
  if (rows > 0) {  // with no rows the gradient is zero, and nothing else is touched
    if (workspace_bytes < p.total) return err.fail(LSAM_ERR_WORKSPACE, "workspace smaller than lsam_embed_grad_workspace_bytes()");
    if (reinterpret_cast<uintptr_t>(d_workspace) & 255) return err.fail(LSAM_ERR_WORKSPACE, "workspace not 256-byte aligned");
    pc.need(d_dout, es); pc.need(d_tokens, 4); pc.need(d_workspace, 256);
  }
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  char* ws = static_cast<char*>(d_workspace);
  const EmbedArgs a{d_tokens, rows, n, vocab, grad_stride_k, grad_stride_row, dout_stride_k, dout_stride_row, scale, FastDiv((uint32_t)std::max<int64_t>(1, rows)), K == 1 || dout_stride_k == rows * dout_stride_row};
  const EmbedLists L{reinterpret_cast<uint2*>(ws), reinterpret_cast<uint2*>(ws + p.b), reinterpret_cast<float*>(ws + p.part), reinterpret_cast<uint32_t*>(ws + p.open), p.N, p.width, (int32_t)p.tiles, p.tile};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool vec = rows_aligned(d_dout, es, K, dout_stride_k, rows, dout_stride_row), vec_out = rows_aligned(d_grad, gs, lists, grad_stride_k, vocab, grad_stride_row);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const T* x = static_cast<const T*>(d_dout);
    if (grad_dtype == LSAM_FP32) e = launch_embed_grad<T, float>(x, static_cast<float*>(d_grad), a, p, L, vec, vec_out, accumulate != 0, stream);
    else e = launch_embed_grad<T, T>(x, static_cast<T*>(d_grad), a, p, L, vec, vec_out, accumulate != 0, stream);
  });
  return err.done(e);
}

// ------------------------------------------------------------------------------------------------ residual norms
namespace {

static_assert((int)GATE_COLUMN == (int)LSAM_GATE_COLUMN && (int)GATE_ROW == (int)LSAM_GATE_ROW && (int)GATE_FULL == (int)LSAM_GATE_FULL, "gates");
static_assert((int)ACT_SIGMOID == (int)LSAM_ACT_SIGMOID && (int)ACT_TANH == (int)LSAM_ACT_TANH, "activations");

constexpr lsam_rows kNoRows{nullptr, 0, 0};

// What both calls check of the description; null: fine.
const char* residual_why(const lsam_residual& r) {
  if (!dtype_ok(r.dtype)) return "unknown dtype";
  if (r.K < 0 || r.rows < 0 || r.n < 0 || r.n > kMaxWide) return "need K, rows >= 0 and 0 <= n <= 2^30";
  if (r.gate < LSAM_GATE_NONE || r.gate > LSAM_GATE_FULL) return "unknown gate";
  if (r.act < LSAM_ACT_LINEAR || r.act > LSAM_ACT_TANH) return "unknown act";
  if (r.K > 0 && r.rows > kMaxIndex / r.K) return "K * rows must be below 2^31";
  if (r.K > 65535) return "K must be below 65536";
  if (r.K == 0 || r.rows == 0 || r.n == 0) return nullptr;  // empty tensors have no addresses
  if (!r.branch.d && (r.post || r.gate != LSAM_GATE_NONE)) return "a norm behind the block or a gate needs a branch";
  if (!r.branch.d && !r.pre) return "neither a branch nor a norm is asked for";
  if ((r.gate != LSAM_GATE_NONE) != (r.gates.d != nullptr)) return "a gate and its kind go together";
  if (r.d_post_weight && !r.post) return "d_post_weight without post";
  if (r.d_pre_weight && !r.pre) return "d_pre_weight without pre";
  return nullptr;
}
struct ResidualCheck {
  const lsam_residual& r;
  PtrCheck pc;
  size_t es;
  const char* why = nullptr;
  explicit ResidualCheck(const lsam_residual& res) : r(res), es(dtype_size(res.dtype)) {}
  void rows(const lsam_rows& t, bool written) {
    if (why || !t.d) return;
    pc.optional(t.d, es);
    if (!strides_ok(r.K, t.stride_k, r.rows, t.stride_row, r.n, 1)) why = "a stride is negative or a tensor is too large";
    else if (r.rows > 1 && t.stride_row > kMaxIndex) why = "row strides must be below 2^31";
    else if (written && !disjoint(r.K, t.stride_k, r.rows, t.stride_row, r.n, 1)) why = "elements of a result share an address or interleave";
  }
  void vector(const void* p, int64_t stride_k) {
    if (why || !p) return;
    pc.optional(p, 4);
    if (!strides_ok(r.K, stride_k, r.n, 1, 1, 0)) why = "a stride is negative or a tensor is too large";
  }
  void inputs() {
    rows(r.branch, false);
    if (r.gate == LSAM_GATE_FULL) rows(r.gates, false);
    else if (r.gate == LSAM_GATE_COLUMN) vector(r.gates.d, r.gates.stride_k);
    else pc.optional(r.gates.d, 4);
    vector(r.d_post_weight, r.post_weight_stride_k);
    vector(r.d_pre_weight, r.pre_weight_stride_k);
  }
  // vectors: every row starts on a 16-byte boundary and holds whole vectors
  bool aligned(const lsam_rows& t) const { return !t.d || (r.n * (int64_t)es % 16 == 0 && rows_aligned(t.d, es, r.K, t.stride_k, r.rows, t.stride_row)); }
  const char* failed() const { return why ? why : pc.why; }
};
template <typename T>
RowsOf<T> rows_of(const lsam_rows& t, const lsam_residual& r) { return {static_cast<T*>(t.d), t.stride_k, r.rows > 1 ? (uint32_t)t.stride_row : 0u}; }

// A warp per row up to four vectors a lane, then as many threads as hold two vectors each; rows longer than 1024 threads hold are read again for each reduction.
template <typename T, bool VEC, int FORM>
cudaError_t launch_residual_norm(const NormArgs<T>& a, cudaStream_t stream) {
  constexpr int E = 2 * vec_n<T>();
  const auto go = [&](auto kern, int threads, int rows, int per_sm, int smem) {
    if (smem > 40 * 1024) {  // beside what is static
      const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e != cudaSuccess) return e;
    }
    kern<<<(unsigned)std::min<int64_t>(ceil_div(a.total, rows), 148 * per_sm), threads, smem, stream>>>(a);
    return cudaPeekAtLastError();
  };
  if (a.n <= 32 * E) return go(residual_norm_kernel<T, 32, E, VEC, FORM>, 128, 4, 8, norm_ring<T, E, VEC>(32));
  if (a.n <= 64 * E) return go(residual_norm_kernel<T, 32, 2 * E, VEC, FORM>, 128, 4, 4, norm_ring<T, 2 * E, VEC>(32));
  if (a.n <= 128 * E) return go(residual_norm_kernel<T, 128, E, VEC, FORM>, 128, 1, 8, norm_ring<T, E, VEC>(128));
  if (a.n <= 256 * E) return go(residual_norm_kernel<T, 256, E, VEC, FORM>, 256, 1, 4, norm_ring<T, E, VEC>(256));
  if (a.n <= 512 * E) return go(residual_norm_kernel<T, 512, E, VEC, FORM>, 512, 1, 2, norm_ring<T, E, VEC>(512));
  if (a.n <= 1024 * E) return go(residual_norm_kernel<T, 1024, E, VEC, FORM>, 1024, 1, 1, norm_ring<T, E, VEC>(1024));
  residual_norm_long_kernel<T><<<a.total, 1024, 0, stream>>>(a);
  return cudaPeekAtLastError();
}

}  // namespace

extern "C" int lsam_residual_norm(const lsam_residual* r, const lsam_rows* x, const lsam_rows* out, const lsam_rows* normed, float* d_rstd_post, float* d_rstd_pre,
                                  void* cuda_stream, char* h_err, size_t h_err_len) {
  const Err err("lsam_residual_norm", h_err, h_err_len);
  if (!r || !x) return err.fail(LSAM_ERR_INVALID, "a required pointer is NULL");
  if (const char* why = residual_why(*r)) return err.fail(LSAM_ERR_INVALID, why);
  if (!(r->eps > 0.f)) return err.fail(LSAM_ERR_INVALID, "eps must be positive");
  if (r->K == 0 || r->rows == 0 || r->n == 0) return LSAM_OK;
  const lsam_rows o = out ? *out : kNoRows, u = normed ? *normed : kNoRows;
  if (!x->d || (r->branch.d && !o.d) || (r->pre && !u.d)) return err.fail(LSAM_ERR_INVALID, "a required pointer is NULL");
  ResidualCheck ck(*r);
  ck.inputs();
  ck.rows(*x, false);
  if (r->branch.d) ck.rows(o, true);
  if (r->pre) ck.rows(u, true);
  ck.pc.optional(d_rstd_post, 4);
  ck.pc.optional(d_rstd_pre, 4);
  if (const char* why = ck.failed()) return err.fail(LSAM_ERR_INVALID, why);
  const bool vec = ck.aligned(*x) && ck.aligned(r->branch) && (r->gate != LSAM_GATE_FULL || ck.aligned(r->gates)) && (!r->branch.d || ck.aligned(o)) && (!r->pre || ck.aligned(u));
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(r->dtype, [&](auto t) {
    using T = decltype(t);
    const bool full = r->gate == LSAM_GATE_FULL;
    const NormArgs<T> a{rows_of<const T>(*x, *r), rows_of<const T>(r->branch, *r), rows_of<const T>(full ? r->gates : kNoRows, *r), rows_of<T>(o, *r), rows_of<T>(u, *r),
                        full ? nullptr : static_cast<const float*>(r->gates.d), r->d_post_weight, r->d_pre_weight, r->gates.stride_k, r->post_weight_stride_k,
                        r->pre_weight_stride_k, d_rstd_post, d_rstd_pre, r->rows, r->n, FastDiv((uint32_t)r->rows), (uint32_t)(r->K * r->rows), r->post, r->pre, r->gate,
                        r->act, r->alpha, r->beta, r->eps, (float)(1.0 / (double)r->n)};
    if (vec && full && r->post && r->pre) e = launch_residual_norm<T, true, FORM_FULL>(a, stream);
    else e = vec ? launch_residual_norm<T, true, FORM_ANY>(a, stream) : launch_residual_norm<T, false, FORM_ANY>(a, stream);
  });
  return err.done(e);
}

namespace {

// Up to 32768 columns one kernel does it all, 512 threads on an SM, each block (or cluster of blocks, past 4096 columns) walking an equal share of the rows;
// longer rows take two passes over strips of rows of one worker, about four blocks of 256 threads on every SM.
struct NormGradPlan {
  int threads, ranks;  // a row's threads in a block (0: two passes), blocks of a cluster
  int64_t per, ld_part, strip, strips, blocks, slots;
  size_t part, total;
};
NormGradPlan norm_grad_plan(int32_t dtype, int32_t K, int64_t rows, int64_t n) {
  NormGradPlan p{};
  p.ld_part = round_up(n, 8);
  if (n <= 4096 * kGradRanks) {
    p.threads = n <= 256 ? 32 : n <= 1024 ? 128 : n <= 2048 ? 256 : 512;
    p.ranks = 1;
    while ((int64_t)p.ranks * 4096 < n) p.ranks *= 2;
    p.per = round_up(ceil_div(n, p.ranks), 8);
    p.ranks = (int)ceil_div(n, p.per);
    const int64_t per_sm = p.threads == 32 ? 4 : 512 / p.threads, turns = p.threads == 32 ? 4 : 1;
    p.strip = std::max(turns, round_up(ceil_div(K * rows, per_sm * (148 / p.ranks)), turns));
    p.blocks = ceil_div(K * rows, p.strip);
    p.slots = p.blocks + K;
  } else {
    const int64_t chunks = ceil_div(n, 256 * (dtype == LSAM_FP32 ? 4 : 8)), want = std::max<int64_t>(1, 4 * 148 / (chunks * K));
    p.strip = ceil_div(rows, std::min(want, rows));
    p.strips = ceil_div(rows, p.strip);
    p.slots = K * p.strips;
    p.part = (size_t)round_up(8 * K * rows, 256);
  }
  p.total = p.part + (size_t)round_up(12 * p.slots * p.ld_part, 256);
  return p;
}

}  // namespace

extern "C" size_t lsam_residual_norm_grad_workspace_bytes(int32_t dtype, int32_t K, int64_t rows, int64_t n) {
  if (!dtype_ok(dtype) || K < 1 || K > 65535 || rows < 1 || rows > kMaxIndex / K || n < 1 || n > kMaxWide) return 0;
  return norm_grad_plan(dtype, K, rows, n).total;
}

namespace {

int residual_norm_grad(const Err& err, const lsam_residual* r, const lsam_rows* out, const float* d_rstd_post, const float* d_rstd_pre, const lsam_rows* dout, const lsam_rows* dnormed,
                       const lsam_rows* dx, const lsam_rows* dbranch, const lsam_rows* dgate, float* d_dpost_weight, float* d_dpre_weight, void* d_workspace, size_t workspace_bytes,
                       bool starved, void* cuda_stream) {
  if (!r) return err.fail(LSAM_ERR_INVALID, "a required pointer is NULL");
  if (const char* why = residual_why(*r)) return err.fail(LSAM_ERR_INVALID, why);
  const lsam_rows y = out ? *out : kNoRows, gy = dout ? *dout : kNoRows, gu = dnormed ? *dnormed : kNoRows, ox = dx ? *dx : kNoRows, ob = dbranch ? *dbranch : kNoRows,
                  oz = dgate ? *dgate : kNoRows;
  if (gu.d && !r->pre) return err.fail(LSAM_ERR_INVALID, "dnormed without pre");
  if (ob.d && !r->branch.d && r->rows > 0 && r->K > 0) return err.fail(LSAM_ERR_INVALID, "dbranch without a branch");
  if (oz.d && r->gate == LSAM_GATE_NONE) return err.fail(LSAM_ERR_INVALID, "dgate without a gate");
  if (d_dpost_weight && !r->post) return err.fail(LSAM_ERR_INVALID, "d_dpost_weight without post");
  if (d_dpre_weight && !r->pre) return err.fail(LSAM_ERR_INVALID, "d_dpre_weight without pre");
  if (r->n == 0) {  // rows of no columns: sums over them are zeros
    if (r->gate != LSAM_GATE_ROW || !oz.d || r->K == 0 || r->rows == 0) return LSAM_OK;
    PtrCheck pc;
    pc.need(oz.d, 4);
    if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
    return err.done(cudaMemsetAsync(oz.d, 0, (size_t)4 * r->K * r->rows, reinterpret_cast<cudaStream_t>(cuda_stream)));
  }
  // without dnormed the norm in front of the next block has no part in the gradient
  const bool pre = r->pre && gu.d;
  ResidualCheck ck(*r);
  const bool full = r->gate == LSAM_GATE_FULL, empty = r->rows == 0 || r->K == 0;  // the sums over no rows are zeros
  if (empty && !d_dpre_weight && !d_dpost_weight && !(r->gate == LSAM_GATE_COLUMN && oz.d)) return LSAM_OK;
  if (!empty) {
    if (!gy.d && !gu.d) return err.fail(LSAM_ERR_INVALID, "neither dout nor dnormed is given");
    if ((pre && (!y.d || !d_rstd_pre)) || (r->post && !d_rstd_post)) return err.fail(LSAM_ERR_INVALID, "a required pointer is NULL");
    ck.inputs();
    if (pre) { ck.rows(y, false); ck.rows(gu, false); ck.pc.need(d_rstd_pre, 4); }
    if (r->post) ck.pc.need(d_rstd_post, 4);
    ck.rows(gy, false); ck.rows(ox, true); ck.rows(ob, true);
    if (full) ck.rows(oz, true);
  }
  if (r->gate == LSAM_GATE_COLUMN || (r->gate == LSAM_GATE_ROW && !empty)) ck.pc.optional(oz.d, 4);
  ck.pc.optional(d_dpost_weight, 4);
  ck.pc.optional(d_dpre_weight, 4);
  NormGradPlan p{};
  if (!empty) {
    p = norm_grad_plan(r->dtype, r->K, r->rows, r->n);
    if (starved && (r->dtype != LSAM_FP32 || p.ranks < 2)) return err.fail(LSAM_ERR_INVALID, "these rows are not shared by a cluster of blocks, or not fp32");
    if (workspace_bytes < p.total) return err.fail(LSAM_ERR_WORKSPACE, "workspace smaller than lsam_residual_norm_grad_workspace_bytes()");
    if (reinterpret_cast<uintptr_t>(d_workspace) & 255) return err.fail(LSAM_ERR_WORKSPACE, "workspace not 256-byte aligned");
    ck.pc.need(d_workspace, 256);
  }
  if (const char* why = ck.failed()) return err.fail(LSAM_ERR_INVALID, why);
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  char* ws = static_cast<char*>(d_workspace);
  // column sums that are wanted, in the order of their places
  NormSumArgs sum{reinterpret_cast<const float*>(ws + p.part), {}, {}, r->n, r->rows, p.strip, p.ld_part, (int32_t)p.strips, 0, r->K};
  const auto want = [&](float* to, int64_t stride_k) {
    if (!to) return 0;
    sum.to[sum.which] = to;
    sum.shared[sum.which] = stride_k == 0 || r->K == 1;
    return ++sum.which;
  };
  const int want_pre = want(d_dpre_weight, r->pre_weight_stride_k), want_post = want(d_dpost_weight, r->post_weight_stride_k);
  const int want_gate = want(r->gate == LSAM_GATE_COLUMN ? static_cast<float*>(oz.d) : nullptr, r->gates.stride_k);
  if (!empty) {
    by_dtype(r->dtype, [&](auto t) {
      using T = decltype(t);
      const bool needs_means = p.threads == 0 && (pre || r->post || (r->gate == LSAM_GATE_ROW && oz.d));
      const NormGradArgs<T> a{rows_of<const T>(y, *r), rows_of<const T>(r->branch, *r), rows_of<const T>(full ? r->gates : kNoRows, *r), rows_of<const T>(gy, *r), rows_of<const T>(gu, *r),
                              rows_of<T>(ox, *r), rows_of<T>(ob, *r), rows_of<T>(full ? oz : kNoRows, *r), full ? nullptr : static_cast<const float*>(r->gates.d), r->d_post_weight,
                              r->d_pre_weight, d_rstd_post, d_rstd_pre, r->gates.stride_k, r->post_weight_stride_k, r->pre_weight_stride_k,
                              r->gate == LSAM_GATE_ROW ? static_cast<float*>(oz.d) : nullptr, needs_means ? reinterpret_cast<float2*>(ws) : nullptr,
                              reinterpret_cast<float*>(ws + p.part), r->rows, r->n, p.strip, p.ld_part, p.per, FastDiv((uint32_t)r->rows), (uint32_t)(r->K * r->rows), (int32_t)p.strips, sum.which,
                              want_pre, want_post, want_gate, r->post, pre, r->gate, r->act, r->alpha, r->beta, (float)(1.0 / (double)r->n)};
      const bool vec = ck.aligned(y) && ck.aligned(r->branch) && ck.aligned(gy) && ck.aligned(gu) && ck.aligned(ox) && ck.aligned(ob) && (!full || (ck.aligned(r->gates) && ck.aligned(oz)));
      if (p.threads) {
        const auto go = [&](auto kern) {
          cudaLaunchConfig_t cfg = {};
          cudaLaunchAttribute attr[1];
          attr[0].id = cudaLaunchAttributeClusterDimension;
          attr[0].val.clusterDim.x = (unsigned)p.ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
          cfg.gridDim = dim3((unsigned)(p.blocks * p.ranks)); cfg.blockDim = dim3(std::max(128, p.threads)); cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = p.ranks > 1 ? 1 : 0;
          return cudaLaunchKernelEx(&cfg, kern, a);
        };
        if constexpr (std::is_same<T, float>::value) {
          if (starved) {
            e = vec ? go(residual_norm_grad_fused_kernel<T, 512, true, true, FORM_ANY, true>) : go(residual_norm_grad_fused_kernel<T, 512, false, true, FORM_ANY, true>);
            return;
          }
        }
        const auto pick = [&](auto v, auto f) {
          constexpr bool V = decltype(v)::value;
          constexpr int F = decltype(f)::value;
          return p.threads == 32 ? go(residual_norm_grad_fused_kernel<T, 32, V, false, F>) : p.threads == 128 ? go(residual_norm_grad_fused_kernel<T, 128, V, false, F>)
                 : p.threads == 256 ? go(residual_norm_grad_fused_kernel<T, 256, V, false, F>) : p.ranks == 1 ? go(residual_norm_grad_fused_kernel<T, 512, V, false, F>)
                                                                                                          : go(residual_norm_grad_fused_kernel<T, 512, V, true, F>);
        };
        const bool all = pre && r->post && gy.d && ox.d && ob.d && r->gate != LSAM_GATE_ROW && (!full || oz.d);
        const auto form = [&](auto v) {
          return all && full ? pick(v, std::integral_constant<int, FORM_FULL>()) : all ? pick(v, std::integral_constant<int, FORM_COLUMN>()) : pick(v, std::integral_constant<int, FORM_ANY>());
        };
        e = vec ? form(std::true_type()) : form(std::false_type());
        return;
      }
      if (needs_means) {
        residual_norm_grad_rows_kernel<T><<<a.total, 256, 0, stream>>>(a);
        e = cudaPeekAtLastError();
        if (e != cudaSuccess) return;
      }
      const dim3 grid((unsigned)ceil_div(r->n, 256 * (vec ? vec_n<T>() : 4)), (unsigned)p.strips, (unsigned)r->K);
      const auto go = [&](auto kern) { return launch_behind(kern, grid, dim3(256), 0, stream, a); };
      e = vec ? go(residual_norm_grad_kernel<T, true>) : go(residual_norm_grad_kernel<T, false>);
    });
  }
  if (e == cudaSuccess && sum.which > 0) {
    const bool each = (!sum.shared[0]) || (sum.which > 1 && !sum.shared[1]) || (sum.which > 2 && !sum.shared[2]);
    const dim3 grid((unsigned)ceil_div(r->n, 128), (unsigned)sum.which, each ? (unsigned)std::max(1, r->K) : 1u);
    e = launch_behind(residual_norm_grad_sum_kernel, grid, dim3(32, kNormSumLanes), 0, stream, sum);
  }
  return err.done(e);
}

}  // namespace

extern "C" int lsam_residual_norm_grad(const lsam_residual* r, const lsam_rows* out, const float* d_rstd_post, const float* d_rstd_pre, const lsam_rows* dout, const lsam_rows* dnormed,
                                       const lsam_rows* dx, const lsam_rows* dbranch, const lsam_rows* dgate, float* d_dpost_weight, float* d_dpre_weight, void* d_workspace,
                                       size_t workspace_bytes, void* cuda_stream, char* h_err, size_t h_err_len) {
  return residual_norm_grad(Err("lsam_residual_norm_grad", h_err, h_err_len), r, out, d_rstd_post, d_rstd_pre, dout, dnormed, dx, dbranch, dgate, d_dpost_weight, d_dpre_weight, d_workspace,
                            workspace_bytes, false, cuda_stream);
}

extern "C" int lsam_selftest_residual_wait(const lsam_residual* r, const lsam_rows* out, const float* d_rstd_post, const float* d_rstd_pre, const lsam_rows* dout, const lsam_rows* dnormed,
                                           const lsam_rows* dx, const lsam_rows* dbranch, const lsam_rows* dgate, float* d_dpost_weight, float* d_dpre_weight, void* d_workspace,
                                           size_t workspace_bytes, void* cuda_stream, char* h_err, size_t h_err_len) {
  return residual_norm_grad(Err("lsam_selftest_residual_wait", h_err, h_err_len), r, out, d_rstd_post, d_rstd_pre, dout, dnormed, dx, dbranch, dgate, d_dpost_weight, d_dpre_weight,
                            d_workspace, workspace_bytes, true, cuda_stream);
}

// ------------------------------------------------------------------------------------------------ orthogonalisation
namespace {

constexpr int64_t kMaxSide = (int64_t)1 << 20;

bool ortho_sizes_ok(int32_t K, int64_t rows, int64_t cols) { return K >= 1 && K <= 65535 && rows >= 1 && cols >= 1 && rows <= kMaxSide && cols <= kMaxSide; }

struct OrthoPlan {
  int64_t m, n, ldm, ldn, chunk;
  int chunks, splits;
  size_t x, y, a, p, part, total;
};
OrthoPlan ortho_plan(int32_t K, int64_t rows, int64_t cols) {
  OrthoPlan q{};
  q.m = std::min(rows, cols);
  q.n = std::max(rows, cols);
  q.ldm = round_up(q.m, 8);
  q.ldn = round_up(q.n, 8);
  // partial sums of squares: no more than occupy the machine eight times
  q.chunk = kNsNorm * ceil_div(rows * cols, kNsNorm * std::max<int64_t>(1, 8 * 148 / K));
  q.chunks = (int)ceil_div(rows * cols, q.chunk);
  if (q.m <= kNsSmall) return q;  // one launch, no workspace
  const int64_t wide = round_up(4 * (int64_t)K * q.m * q.ldn, 256), square = round_up(4 * (int64_t)K * q.m * q.ldm, 256);  // two fp16 planes
  q.x = (size_t)round_up(8 * (int64_t)K * q.chunks, 256);
  q.y = q.x + (size_t)wide;
  q.a = q.y + (size_t)wide;
  q.p = q.a + (size_t)square;
  q.part = q.p + (size_t)square;
  q.splits = ns_splits(K, q.m, q.n);
  q.total = q.part + (q.splits > 1 ? (size_t)round_up(4 * (int64_t)K * q.splits * q.m * q.ldm, 256) : 0);
  return q;
}

// The largest |p(s)|, p(s) = a s + b s^3 + c s^5, over 0 <= s <= top: at the end, or where p' = a + 3 b s^2 + 5 c s^4 vanishes.
double ortho_reach(double a, double b, double c, double top) {
  const auto at = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
  double best = at(top);
  const auto root = [&](double u) {
    if (u > 0.0 && u < top * top) best = std::max(best, at(std::sqrt(u)));
  };
  // 5 c u^2 + 3 b u + a = 0, the roots as q / (5 c) and a / q: neither is lost beside a small c (nor needs one)
  const double d = 9.0 * b * b - 20.0 * a * c;
  if (d >= 0.0) {
    const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));
    if (c != 0.0) root(q / (5.0 * c));
    if (q != 0.0) root(a / q);
  }
  return best;
}

// The largest |b u + c u^2| over 0 <= u <= top: what the eigenvalues of P are bounded by.
double ortho_reach_square(double b, double c, double top) {
  double best = std::fabs(top * (b + c * top));
  if (c != 0.0) {
    const double u = -b / (2.0 * c);
    if (u > 0.0 && u < top) best = std::max(best, std::fabs(u * (b + c * u)));
  }
  return best;
}
// The power of two that brings what is bounded by `bound` to at most 2^14, with room for the roundings of what is bounded by one.
int ortho_exponent(double bound) {
  int e = 0;
  std::frexp(std::max(bound, 1e-30), &e);  // bound < 2^e
  return std::max(-60, std::min(60, 14 - e));
}

}  // namespace

extern "C" size_t lsam_orthogonalize_workspace_bytes(int32_t dtype, int32_t K, int64_t rows, int64_t cols) {
  if (!dtype_ok(dtype) || !ortho_sizes_ok(K, rows, cols)) return 0;
  return ortho_plan(K, rows, cols).total;
}

namespace {

int orthogonalize(const Err& err, const void* d_g, int32_t dtype, int32_t K, int64_t rows, int64_t cols, int64_t stride_k, int64_t stride_row, int64_t stride_col, int32_t steps, float a, float b,
                  float c, float scale, float eps, void* d_out, int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_col, void* d_workspace, size_t workspace_bytes, bool starved,
                  void* cuda_stream) {
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (K < 0 || rows < 0 || cols < 0 || K > 65535 || rows > kMaxSide || cols > kMaxSide) return err.fail(LSAM_ERR_INVALID, "need 0 <= K <= 65535 and 0 <= rows, cols <= 2^20");
  if (steps < 0 || steps > 32) return err.fail(LSAM_ERR_INVALID, "steps outside 0 .. 32");
  if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(scale)) return err.fail(LSAM_ERR_INVALID, "eps must be finite and not negative, scale finite");
  // the last product's sums carry the planes' powers of two, 2^33 at most, and are freed of them by one fp32 factor together with scale
  if (scale != 0.f && std::fabs(scale) < 0x1p-90f) return err.fail(LSAM_ERR_INVALID, "scale must be zero or at least 2^-90");
  // with |a| < 1 a step shrinks small singular values, and the next ones find them below what two fp16 planes hold of their common bound
  if (steps > 0 && !(std::fabs(a) >= 1.f)) return err.fail(LSAM_ERR_INVALID, "|a| must be at least 1");
  double reach = 1.0;
  for (int32_t t = 0; t < steps; ++t) {
    reach = ortho_reach(a, b, c, reach);
    if (!(reach < 1024.0)) return err.fail(LSAM_ERR_INVALID, "with these coefficients singular values are not bounded by 2^10");
  }
  if (K == 0 || rows == 0 || cols == 0) return LSAM_OK;
  if (!strides_ok(K, stride_k, rows, stride_row, cols, stride_col) || !strides_ok(K, out_stride_k, rows, out_stride_row, cols, out_stride_col))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or a tensor is too large");
  if (!disjoint(K, out_stride_k, rows, out_stride_row, cols, out_stride_col)) return err.fail(LSAM_ERR_INVALID, "elements of the output share an address or interleave");
  const OrthoPlan q = ortho_plan(K, rows, cols);
  if (starved && (dtype != LSAM_FP32 || q.m <= kNsSmall || steps == 0)) return err.fail(LSAM_ERR_INVALID, "these matrices do not go to the tensor cores, or are not fp32");
  if (workspace_bytes < q.total) return err.fail(LSAM_ERR_WORKSPACE, "workspace smaller than lsam_orthogonalize_workspace_bytes()");
  if (q.total && reinterpret_cast<uintptr_t>(d_workspace) & 255) return err.fail(LSAM_ERR_WORKSPACE, "workspace not 256-byte aligned");
  const size_t es = dtype_size(dtype);
  PtrCheck pc;
  pc.need(d_g, es); pc.need(d_out, es);
  if (q.total) pc.need(d_workspace, 256);
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  char* ws = static_cast<char*>(d_workspace);
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const T* g = static_cast<const T*>(d_g);
    T* out = static_cast<T*>(d_out);
    const bool tall = rows > cols;
    const int64_t m = q.m, n = q.n, oi = tall ? out_stride_col : out_stride_row, oj = tall ? out_stride_row : out_stride_col;
    if (m <= kNsSmall) {
      const int64_t si = tall ? stride_col : stride_row, sj = tall ? stride_row : stride_col;
      const auto small = [&](auto kern, int smem) {
        // blocks of a cluster: slices of at least 128 columns, no more blocks than occupy the machine twice
        int ranks = 8;
        while (ranks > 1 && (n < 128 * ranks || (int64_t)K * ranks > 2 * 148)) ranks /= 2;
        cudaError_t f = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (f != cudaSuccess) return f;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3((unsigned)(K * ranks)); cfg.blockDim = dim3(256); cfg.dynamicSmemBytes = (size_t)smem; cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, kern, g, stride_k, si, sj, (int)m, n, ceil_div(n, (int64_t)ranks), steps, (double)a, (double)b, (double)c, (double)scale, (double)eps, out,
                                  out_stride_k, oi, oj);
      };
      e = m <= 16 ? small(ns_small_kernel<T, 1>, ns_small_smem<1>()) : small(ns_small_kernel<T, 2>, ns_small_smem<2>());
      return;
    }
    double* part = reinterpret_cast<double*>(ws);
    NsPlanes x{reinterpret_cast<fp16*>(ws + q.x), m * q.ldn, q.ldn}, y{reinterpret_cast<fp16*>(ws + q.y), m * q.ldn, q.ldn};
    const NsPlanes A{reinterpret_cast<fp16*>(ws + q.a), m * q.ldm, q.ldm}, P{reinterpret_cast<fp16*>(ws + q.p), m * q.ldm, q.ldm};
    const bool along_rows = stride_col <= stride_row;
    const int64_t inner = along_rows ? cols : rows, so = along_rows ? stride_row : stride_col, unit = along_rows ? stride_col : stride_row;
    // whole vectors along the contiguous index
    const bool vec = (unit == 1 || inner == 1) && inner % vec_n<T>() == 0 && rows_aligned(d_g, es, K, stride_k, along_rows ? rows : cols, so);
    if (vec) {
      ns_norm_kernel<T, true><<<dim3((unsigned)q.chunks, (unsigned)K), 256, 0, stream>>>(g, stride_k, so, unit, inner / vec_n<T>(), rows * cols / vec_n<T>(), q.chunk / vec_n<T>(), part);
    } else {
      ns_norm_kernel<T, false><<<dim3((unsigned)q.chunks, (unsigned)K), 256, 0, stream>>>(g, stride_k, so, unit, inner, rows * cols, q.chunk, part);
    }
    if ((e = cudaPeekAtLastError()) != cudaSuccess) return;
    const int64_t si = tall ? stride_col : stride_row, sj = tall ? stride_row : stride_col;
    if (steps == 0) {
      ns_only_norm_kernel<T><<<dim3((unsigned)ceil_div(m * n, 256), (unsigned)K), 256, 0, stream>>>(g, stride_k, si, sj, m, n, part, q.chunks, eps, scale, out, out_stride_k, oi, oj);
      e = cudaPeekAtLastError();
      return;
    }
    double top = 1.0;  // the largest singular value that X can have
    int ex = ortho_exponent(top);
    if (vec && sj == 1 && n % 8 == 0)
      e = launch_behind(ns_start_rows_kernel<T>, dim3((unsigned)ceil_div(m * n / 8, 256), (unsigned)K), dim3(256), 0, stream, g, stride_k, si, (uint32_t)(n / 8), m * n / 8,
                        static_cast<const double*>(part), q.chunks, eps, std::ldexp(1.0, ex), x);
    else e = launch_behind(ns_start_kernel<T>, dim3((unsigned)ceil_div(n, 64), (unsigned)ceil_div(m, 64), (unsigned)K), dim3(256), 0, stream, g, stride_k, si, sj, m, n,
                      static_cast<const double*>(part), q.chunks, eps, std::ldexp(1.0, ex), x);
    for (int32_t s = 0; s < steps && e == cudaSuccess; ++s) {
      const double next = ortho_reach(a, b, c, top);
      const int ea = ortho_exponent(top * top), ep = ortho_exponent(ortho_reach_square(b, c, top * top) + std::fabs((double)a)), en = ortho_exponent(next);
      const auto two = [](int v) { return (float)std::ldexp(1.0, v); };
      NsGemm w{};
      w.m = w.n = (int)m; w.inner = (int)n;
      w.f = two(ea - 2 * ex);
      w.out = A;
      if (q.splits > 1) {
        NsGemm v = w;
        v.splits = q.splits; v.split_blocks = (int)ceil_div(ceil_div(n, (int64_t)kNsK), (int64_t)q.splits);
        v.f = 1.f;
        float* sums = reinterpret_cast<float*>(ws + q.part);
        v.final_out = sums; v.ok = m * q.ldm; v.oi = q.ldm; v.oj = 1;
        e = ns_launch<float, NS_PART>(x, x, v, K, starved, stream);
        if (e == cudaSuccess)
          e = launch_behind(ns_join_kernel, dim3((unsigned)ceil_div(m * q.ldm, 1024), (unsigned)K), dim3(256), 0, stream, static_cast<const float*>(sums), q.splits, m, A, w.f);
      } else {
        e = ns_launch<fp16, NS_GRAM>(x, x, w, K, starved, stream);
      }
      if (e != cudaSuccess) return;
      w.inner = (int)m;
      // the term a X of the last product is the diagonal of P
      w.f = c * two(ep - 2 * ea); w.h = b * two(ep - ea); w.diagonal = a * two(ep);
      w.other = A; w.out = P;
      e = ns_launch<fp16, NS_SQUARE>(A, A, w, K, starved, stream);
      if (e != cudaSuccess) return;
      w.n = (int)n;
      w.out = y;
      if (s + 1 < steps) {
        w.f = two(en - ep - ex);
        e = ns_launch<fp16, NS_APPLY>(P, x, w, K, starved, stream);
      } else {
        w.f = scale * two(-ep - ex);
        w.final_out = out; w.ok = out_stride_k; w.oi = oi; w.oj = oj;
        e = ns_launch<T, NS_FINAL>(P, x, w, K, starved, stream);
      }
      std::swap(x, y);
      top = next; ex = en;
    }
  });
  return err.done(e);
}

}  // namespace

extern "C" int lsam_orthogonalize(const void* d_g, int32_t dtype, int32_t K, int64_t rows, int64_t cols, int64_t stride_k, int64_t stride_row, int64_t stride_col, int32_t steps, float a,
                                  float b, float c, float scale, float eps, void* d_out, int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_col, void* d_workspace,
                                  size_t workspace_bytes, void* cuda_stream, char* h_err, size_t h_err_len) {
  return orthogonalize(Err("lsam_orthogonalize", h_err, h_err_len), d_g, dtype, K, rows, cols, stride_k, stride_row, stride_col, steps, a, b, c, scale, eps, d_out, out_stride_k, out_stride_row,
                       out_stride_col, d_workspace, workspace_bytes, false, cuda_stream);
}

extern "C" int lsam_selftest_orthogonalize_wait(const void* d_g, int32_t dtype, int32_t K, int64_t rows, int64_t cols, int64_t stride_k, int64_t stride_row, int64_t stride_col, int32_t steps,
                                                float a, float b, float c, float scale, float eps, void* d_out, int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_col,
                                                void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* h_err, size_t h_err_len) {
  return orthogonalize(Err("lsam_selftest_orthogonalize_wait", h_err, h_err_len), d_g, dtype, K, rows, cols, stride_k, stride_row, stride_col, steps, a, b, c, scale, eps, d_out, out_stride_k,
                       out_stride_row, out_stride_col, d_workspace, workspace_bytes, true, cuda_stream);
}
