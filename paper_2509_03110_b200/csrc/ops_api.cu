// ops_api.cu -- host side of the operators around a classifier's head (include/lsam.h, last section): argument checks and
// launches.  Nothing here allocates, synchronises or keeps state between calls.
#include "lsam.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <type_traits>
#include <utility>

#include "common.cuh"
#include "dropout.cuh"
#include "head_ops.cuh"
#include "head_score.cuh"
#include "head_tcgen05.cuh"

using namespace lsam;

namespace {

struct Err {
  const char* fn;
  char* buf;
  size_t len;
  Err(const char* f, char* b, size_t n) : fn(f), buf(b), len(n) {
    if (buf && len > 0) buf[0] = 0;
  }
  int fail(int code, const char* msg) const {
    if (buf && len > 0) std::snprintf(buf, len, "%s: %s", fn, msg);
    return code;
  }
  int done(cudaError_t e) const {
    if (e == cudaSuccess) return LSAM_OK;
    (void)cudaGetLastError();
    if (buf && len > 0) std::snprintf(buf, len, "%s: launch failed: %s", fn, cudaGetErrorString(e));
    return LSAM_ERR_CUDA;
  }
};

size_t dtype_size(int32_t d) { return d == LSAM_FP32 ? 4 : 2; }
bool dtype_ok(int32_t d) { return d == LSAM_FP32 || d == LSAM_BF16 || d == LSAM_FP16; }

// Every pointer a kernel will touch is memory of the current device, aligned to its elements.
struct PtrCheck {
  int dev = -1;
  const char* why = nullptr;
  PtrCheck() {
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); why = "no current device"; }
  }
  void need(const void* p, size_t align) {
    if (why) return;
    if (!p) { why = "a required pointer is NULL"; return; }
    optional(p, align);
  }
  void optional(const void* p, size_t align) {
    if (why || !p) return;
    if (reinterpret_cast<uintptr_t>(p) % align) { why = "a pointer is not aligned to its element type"; return; }
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) { (void)cudaGetLastError(); why = "a pointer is not device memory"; return; }
    if (a.type == cudaMemoryTypeManaged) return;
    if (a.type != cudaMemoryTypeDevice) why = "a pointer is not device memory";
    else if (a.device != dev) why = "a pointer belongs to another device than the current one";
  }
};

constexpr int64_t kMaxIndex = ((int64_t)1 << 31) - 1, kMaxHead = (int64_t)1 << 30;

// extents n0 x n1 x n2 with element strides s0, s1, s2: every offset fits a signed 64-bit byte count
bool strides_ok(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  if (s0 < 0 || s1 < 0 || s2 < 0) return false;
  const __int128 last = (__int128)(n0 - 1) * s0 + (__int128)(n1 - 1) * s1 + (__int128)(n2 - 1) * s2;
  return last < ((__int128)1 << 60);
}

// No two elements at one address: in the order of their strides, every dimension steps over all that the smaller ones span.
bool disjoint(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  std::pair<int64_t, int64_t> d[3] = {{s0, n0}, {s1, n1}, {s2, n2}};
  std::sort(d, d + 3);
  __int128 span = 1;
  for (const auto& e : d) {
    if (e.second <= 1) continue;
    if (e.first < span) return false;
    span += (__int128)e.first * (e.second - 1);
  }
  return true;
}

template <class F>
void by_dtype(int32_t d, F&& f) {
  if (d == LSAM_FP32) f(float());
  else if (d == LSAM_BF16) f(bf16());
  else f(fp16());
}

}  // namespace

namespace {

template <typename T, int NT, int CS>
cudaError_t launch_row(const LogitView<T>& v, const int32_t* labels, const ScoreOut& out, int64_t total, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(total * CS)); cfg.blockDim = dim3(NT); cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = CS > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, logprob_row_kernel<T, NT, CS>, v, labels, out);
}

// Which form a call takes.  Many rows of few classes: a thread per row, from 32768 rows of up to 256 classes with the sample index contiguous (106647
// rows of 95 bf16: 87 us in the feature kernel, 9 with a thread per row; 5 alternatives 40), from 4096 rows of up to 64 contiguous classes (60000 rows
// of 10 fp32: 3 us), unless the alternatives, a walk over the row each, cost more (8192 rows of 64, 8 alternatives: 47 us against a warp's 13).  Other
// sample-contiguous logits go to the feature kernel.  Rows of contiguous classes: a warp per row up to 1024 classes, 128 threads up to 32 KB, 256 beyond;
// rows of 32 KB and more that leave most of the machine idle are split over a cluster of 8 or 4 blocks (4 rows of 131072 bf16, 8 alternatives: 14.4 us
// with one block a row, 8.3 with eight; 64 rows: 14.4, four blocks 10.7).
template <typename T>
cudaError_t launch_scores(const LogitView<T>& v, const int32_t* labels, const ScoreOut& out, int32_t K, cudaStream_t stream) {
  const int64_t total = (int64_t)K * v.rows;
  const bool samples = v.sc != 1 && v.sr == 1 && v.rows > 1;
  const int64_t walks = (int64_t)out.top_k * v.classes;
  if (samples ? total >= 32768 && v.classes <= 256 && walks <= 512 : total >= 4096 && v.classes <= 64 && (out.top_k <= 1 || walks <= 160)) {
    logprob_thread_kernel<T><<<(unsigned)ceil_div(total, 128), 128, 0, stream>>>(v, labels, out, (uint32_t)total);
    return cudaPeekAtLastError();
  }
  if (samples) {
    const int64_t row_blocks = ceil_div(v.rows, feat_rows<T>());
    logprob_feature_kernel<T><<<(unsigned)(K * row_blocks), feat_rows<T>() * kFeatG, 0, stream>>>(v, labels, out, (uint32_t)row_blocks);
    return cudaPeekAtLastError();
  }
  if (v.classes <= kWarpClasses) {
    const int64_t es = sizeof(T);
    const bool vec = v.sc == 1 && reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && (v.rows == 1 || v.sr * es % 16 == 0) && (K == 1 || v.sk * es % 16 == 0);
    const unsigned blocks = (unsigned)ceil_div(total, 8);
    if (vec) logprob_warp_kernel<T, true><<<blocks, 256, 0, stream>>>(v, labels, out, (uint32_t)total);
    else logprob_warp_kernel<T, false><<<blocks, 256, 0, stream>>>(v, labels, out, (uint32_t)total);
    return cudaPeekAtLastError();
  }
  const int64_t bytes = (int64_t)v.classes * sizeof(T);
  if (bytes >= 32768 && total <= 148 / 4) return launch_row<T, 256, 8>(v, labels, out, total, stream);
  if (bytes >= 32768 && total <= 148) return launch_row<T, 256, 4>(v, labels, out, total, stream);
  if (bytes <= 32768) return launch_row<T, 128, 1>(v, labels, out, total, stream);
  return launch_row<T, 256, 1>(v, labels, out, total, stream);
}

}  // namespace

namespace {

int logprob(const Err& err, const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row, int64_t stride_class,
            const int32_t* d_labels, int32_t top_k, float* d_logp, float* d_lse, float* d_lse_low, float* d_entropy, float* d_top_logp, int32_t* d_top_idx, void* cuda_stream) {
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (K < 0 || rows < 0 || classes < 1 || classes > kMaxIndex) return err.fail(LSAM_ERR_INVALID, "need K >= 0, rows >= 0, 1 <= classes < 2^31");
  if (top_k < 0 || top_k > LSAM_TOP_MAX) return err.fail(LSAM_ERR_INVALID, "top_k outside 0 .. LSAM_TOP_MAX");
  if (d_logp && !d_labels) return err.fail(LSAM_ERR_INVALID, "d_logp without d_labels");
  if (K == 0 || rows == 0) return LSAM_OK;
  if (rows > kMaxIndex / K) return err.fail(LSAM_ERR_INVALID, "K * rows must be below 2^31");
  if (!strides_ok(K, stride_k, rows, stride_row, classes, stride_class)) return err.fail(LSAM_ERR_INVALID, "a stride is negative or the tensor is too large");
  PtrCheck pc;
  pc.need(d_logits, dtype_size(dtype));
  pc.optional(d_labels, 4); pc.optional(d_logp, 4); pc.optional(d_lse, 4); pc.optional(d_entropy, 4); pc.optional(d_lse_low, 4);
  if (top_k > 0) { pc.need(d_top_logp, 4); pc.need(d_top_idx, 4); }
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  const ScoreOut out{d_logp, d_lse, d_entropy, d_top_logp, d_top_idx, top_k, d_lse_low};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const LogitView<T> v{static_cast<const T*>(d_logits), rows, stride_k, stride_row, stride_class, (int32_t)classes, FastDiv((uint32_t)rows)};
    e = launch_scores<T>(v, d_labels, out, K, stream);
  });
  return err.done(e);
}

}  // namespace

extern "C" int lsam_logprob(const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row,
                            int64_t stride_class, const int32_t* d_labels, int32_t top_k, float* d_logp, float* d_lse, float* d_entropy,
                            float* d_top_logp, int32_t* d_top_idx, void* cuda_stream, char* h_err, size_t h_err_len) {
  return logprob(Err("lsam_logprob", h_err, h_err_len), d_logits, dtype, K, rows, classes, stride_k, stride_row, stride_class, d_labels, top_k, d_logp, d_lse, nullptr,
                 d_entropy, d_top_logp, d_top_idx, cuda_stream);
}

extern "C" int lsam_logprob_wide(const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row,
                                 int64_t stride_class, const int32_t* d_labels, int32_t top_k, float* d_logp, float* d_lse, float* d_lse_low, float* d_entropy,
                                 float* d_top_logp, int32_t* d_top_idx, void* cuda_stream, char* h_err, size_t h_err_len) {
  return logprob(Err("lsam_logprob_wide", h_err, h_err_len), d_logits, dtype, K, rows, classes, stride_k, stride_row, stride_class, d_labels, top_k, d_logp, d_lse, d_lse_low,
                 d_entropy, d_top_logp, d_top_idx, cuda_stream);
}

namespace {

// Form of a gradient call: vectors along the classes or along the samples where both tensors have that index contiguous and every row of
// the two starts at the same place of a 16-byte vector, single elements in the same order otherwise.
template <typename T, bool TWO>
cudaError_t launch_grad(const LogitView<T>& v, const GradIn& in, const GradOut<T>& o, int32_t K, cudaStream_t stream) {
  const int64_t total = (int64_t)K * v.rows;
  const auto aligned = [](int64_t elems) { return elems * (int64_t)sizeof(T) % 16 == 0; };
  const uintptr_t pi = reinterpret_cast<uintptr_t>(v.p), po = reinterpret_cast<uintptr_t>(o.p);
  if (v.sc != 1 && v.sr == 1 && o.sr == 1 && v.rows > 1) {
    const bool vec = pi % 16 == 0 && po % 16 == 0 && aligned(v.sc) && aligned(o.sc) && (K == 1 || (aligned(v.sk) && aligned(o.sk)));
    const int64_t class_blocks = ceil_div(v.classes, 64), row_blocks = ceil_div(v.rows, vec ? 32 * vec_n<T>() : 32);
    if (class_blocks * row_blocks <= kMaxIndex / K) {
      const unsigned grid = (unsigned)(class_blocks * row_blocks * K);
      if (vec) grad_feature_kernel<T, vec_n<T>(), TWO><<<grid, dim3(32, 8), 0, stream>>>(v, in, o, (uint32_t)row_blocks, (uint32_t)class_blocks);
      else grad_feature_kernel<T, 1, TWO><<<grid, dim3(32, 8), 0, stream>>>(v, in, o, (uint32_t)row_blocks, (uint32_t)class_blocks);
      return cudaPeekAtLastError();
    }
  }
  const bool vec = v.sc == 1 && o.sc == 1 && (pi - po) % 16 == 0 && (v.rows == 1 || aligned(v.sr - o.sr)) && (K == 1 || aligned(v.sk - o.sk));
  const bool unit = v.sc == 1 && o.sc == 1, narrow = v.classes <= 1024;  // narrow: a warp per row
  const auto go = [&](auto kern, int64_t chunk) {
    const int64_t chunks = ceil_div(v.classes, chunk), units = total * chunks, blocks = narrow ? ceil_div(units, 8) : units;
    if (units > kMaxIndex) return cudaErrorInvalidConfiguration;
    kern<<<(unsigned)blocks, 256, 0, stream>>>(v, in, o, FastDiv((uint32_t)chunks), (uint32_t)units);
    return cudaPeekAtLastError();
  };
  const auto pick = [&](auto mode) {
    constexpr int M = decltype(mode)::value;
    return narrow ? go(grad_row_kernel<T, 32, M, TWO>, grad_chunk<T>(M, 32)) : go(grad_row_kernel<T, 256, M, TWO>, grad_chunk<T>(M, 256));
  };
  if (vec) return pick(std::integral_constant<int, GRAD_VECTORS>());
  return unit ? pick(std::integral_constant<int, GRAD_UNIT>()) : pick(std::integral_constant<int, GRAD_ANY>());
}

}  // namespace

namespace {

int logprob_grad(const Err& err, const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row, int64_t stride_class,
                 const int32_t* d_labels, const float* d_lse, const float* d_lse_low, const float* d_entropy, const float* d_dlogp, const float* d_dentropy, void* d_dlogits,
                 int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_class, void* cuda_stream) {
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (K < 0 || rows < 0 || classes < 1 || classes > kMaxIndex) return err.fail(LSAM_ERR_INVALID, "need K >= 0, rows >= 0, 1 <= classes < 2^31");
  if (!d_dlogp && !d_dentropy) return err.fail(LSAM_ERR_INVALID, "neither d_dlogp nor d_dentropy is given");
  if (d_dlogp && !d_labels) return err.fail(LSAM_ERR_INVALID, "d_dlogp without d_labels");
  if (d_dentropy && !d_entropy) return err.fail(LSAM_ERR_INVALID, "d_dentropy without d_entropy");
  if (K == 0 || rows == 0) return LSAM_OK;
  if (rows > kMaxIndex / K) return err.fail(LSAM_ERR_INVALID, "K * rows must be below 2^31");
  if (!strides_ok(K, stride_k, rows, stride_row, classes, stride_class) || !strides_ok(K, out_stride_k, rows, out_stride_row, classes, out_stride_class))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or the tensor is too large");
  if (!disjoint(K, out_stride_k, rows, out_stride_row, classes, out_stride_class)) return err.fail(LSAM_ERR_INVALID, "elements of the gradient share an address or interleave");
  PtrCheck pc;
  pc.need(d_logits, dtype_size(dtype)); pc.need(d_dlogits, dtype_size(dtype)); pc.need(d_lse, 4);
  pc.optional(d_labels, 4); pc.optional(d_entropy, 4); pc.optional(d_dlogp, 4); pc.optional(d_dentropy, 4); pc.optional(d_lse_low, 4);
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  const GradIn in{d_labels, d_lse, d_entropy, d_dlogp, d_dentropy, d_lse_low};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const LogitView<T> v{static_cast<const T*>(d_logits), rows, stride_k, stride_row, stride_class, (int32_t)classes, FastDiv((uint32_t)rows)};
    const GradOut<T> o{static_cast<T*>(d_dlogits), out_stride_k, out_stride_row, out_stride_class};
    e = d_lse_low ? launch_grad<T, true>(v, in, o, K, stream) : launch_grad<T, false>(v, in, o, K, stream);
  });
  return err.done(e);
}

}  // namespace

extern "C" int lsam_logprob_grad(const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row,
                                 int64_t stride_class, const int32_t* d_labels, const float* d_lse, const float* d_entropy, const float* d_dlogp,
                                 const float* d_dentropy, void* d_dlogits, int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_class,
                                 void* cuda_stream, char* h_err, size_t h_err_len) {
  return logprob_grad(Err("lsam_logprob_grad", h_err, h_err_len), d_logits, dtype, K, rows, classes, stride_k, stride_row, stride_class, d_labels, d_lse, nullptr, d_entropy, d_dlogp,
                      d_dentropy, d_dlogits, out_stride_k, out_stride_row, out_stride_class, cuda_stream);
}

extern "C" int lsam_logprob_grad_wide(const void* d_logits, int32_t dtype, int32_t K, int64_t rows, int64_t classes, int64_t stride_k, int64_t stride_row,
                                      int64_t stride_class, const int32_t* d_labels, const float* d_lse, const float* d_lse_low, const float* d_entropy, const float* d_dlogp,
                                      const float* d_dentropy, void* d_dlogits, int64_t out_stride_k, int64_t out_stride_row, int64_t out_stride_class,
                                      void* cuda_stream, char* h_err, size_t h_err_len) {
  return logprob_grad(Err("lsam_logprob_grad_wide", h_err, h_err_len), d_logits, dtype, K, rows, classes, stride_k, stride_row, stride_class, d_labels, d_lse, d_lse_low, d_entropy,
                      d_dlogp, d_dentropy, d_dlogits, out_stride_k, out_stride_row, out_stride_class, cuda_stream);
}

namespace {

// Forms of a head call, by sizes, type and alignment:
//   TENSOR  16-bit operands that TMA takes as they are;
//   GEMV    at most eight rows that TMA does not take (fp32, unaligned): straight from memory to the FMA pipes;
//   TILES   small products: at most kTileSteps steps of kHsK inner indices for every SM's blocks;
//   COPY    the rest: copied into aligned rows (fp32: three bf16 planes), then the tensor cores.
// A step of TILES takes 0.8 to 1.7 us, whatever the rows; COPY has one launch more and moves both matrices.  Measured (us, TILES / COPY), bf16 rows x inner x
// classes: 16 x 20 x 1000 7.4 / 8.9, 300 x 20 x 1000 7.7 / 11.2, 16 x 101 x 70 11.8 / 8.1, 82 x 301 x 1000 24 / 10.7, 82 x 1091 x 70 70 / 11.7, 2000 x 1021 x 16384
// 4297 / 96;  fp32: 40 x 8 x 20001 12 / 33, 101 x 394 x 1722 31 / 19.8;  4 x 4096 x 32768 fp32 in tiles 287, GEMV 102.
enum HeadForm { HEAD_TENSOR, HEAD_GEMV, HEAD_COPY, HEAD_TILES };
constexpr int64_t kTileSteps = 4;
// GEMV and TILES: shares of the classes, enough to occupy the machine, none shorter than what a block takes at a time.
struct SharePlan {
  int splits = 1;
  int64_t per_split = 0;
};
SharePlan share_plan(HeadForm f, int32_t K, int64_t rows, int64_t classes) {
  SharePlan p;
  const int64_t least = f == HEAD_GEMV ? 64 : kHsN, blocks = (int64_t)K * (f == HEAD_GEMV ? 1 : ceil_div(rows, kHsM));
  const int64_t splits = std::min<int64_t>(ceil_div(2 * 148, blocks), ceil_div(classes, least));
  p.per_split = round_up(ceil_div(classes, splits), least);
  p.splits = (int)ceil_div(classes, p.per_split);
  return p;
}
HeadForm head_form(int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes, bool aligned) {
  if (dtype != LSAM_FP32 && aligned) return HEAD_TENSOR;
  if (rows <= kGemvRows && gemv_smem(rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8, inner) <= kGemvSmem) return HEAD_GEMV;
  const SharePlan p = share_plan(HEAD_TILES, K, rows, classes);
  const int64_t waves = ceil_div(K * ceil_div(rows, kHsM) * p.splits, 2 * 148);
  return waves * ceil_div(p.per_split, kHsN) * ceil_div(inner, kHsK) <= kTileSteps ? HEAD_TILES : HEAD_COPY;
}
// The workspace: partial statistics, the labels' logits, and in the COPY form the two matrices.
struct HeadSpace {
  size_t label, h, w, total;
  int64_t pad;
};
// The form of a call and how it is split: `share` for GEMV and TILES, `tile` for the tensor cores.
struct HeadPlan {
  HeadForm form;
  SharePlan share;
  HeadTile tile{};
};
HeadPlan head_plan(int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes, bool aligned) {
  HeadPlan p{head_form(dtype, K, rows, inner, classes, aligned)};
  if (p.form == HEAD_GEMV || p.form == HEAD_TILES) p.share = share_plan(p.form, K, rows, classes);
  else p.tile = ht_plan(K, rows, classes);
  return p;
}
HeadSpace head_space(const HeadPlan& p, int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes, bool shared_w) {
  const HeadForm f = p.form;
  const int64_t parts = f == HEAD_GEMV || f == HEAD_TILES ? p.share.splits : 2 * p.tile.runs;
  const int64_t planes = dtype == LSAM_FP32 ? 3 : 1;
  HeadSpace s;
  s.pad = round_up(inner, 8);
  s.label = (size_t)round_up((int64_t)sizeof(RowStat) * parts * K * rows, 256);
  s.h = s.w = s.total = s.label + (size_t)round_up(4 * (int64_t)K * rows, 256);
  if (f == HEAD_COPY) {
    s.w = s.h + (size_t)round_up(2 * planes * K * rows * s.pad, 256);
    s.total = s.w + (size_t)round_up(2 * planes * (shared_w ? 1 : K) * classes * s.pad, 256);
  }
  return s;
}
bool head_sizes_ok(int32_t K, int64_t rows, int64_t inner, int64_t classes) {
  return K >= 1 && K <= 65535 && rows >= 1 && rows <= 4194240 && rows <= kMaxIndex / K && inner >= 1 && inner <= kMaxHead && classes >= 1 && classes <= kMaxHead;
}

template <typename T>
cudaError_t launch_gemv(const T* h, const T* w, const HeadArgs& a, int32_t K, bool vec, cudaStream_t stream) {
  const int R = a.rows <= 1 ? 1 : a.rows <= 2 ? 2 : a.rows <= 4 ? 4 : 8;
  const int smem = (int)gemv_smem(R, a.inner);
  const auto go = [&](auto kern) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemvSmem);
    if (e != cudaSuccess) return e;
    kern<<<dim3((unsigned)a.parts, 1, (unsigned)K), 256, smem, stream>>>(h, w, a);
    return cudaPeekAtLastError();
  };
  const auto pick = [&](auto v) {
    constexpr bool V = decltype(v)::value;
    return R == 1 ? go(head_gemv_kernel<T, 1, V>) : R == 2 ? go(head_gemv_kernel<T, 2, V>) : R == 4 ? go(head_gemv_kernel<T, 4, V>) : go(head_gemv_kernel<T, 8, V>);
  };
  return vec ? pick(std::true_type()) : pick(std::false_type());
}

// The widest group of lanes that leaves few of them idle at the end of a row.
template <typename T, typename D>
cudaError_t launch_copy(CopySide h, CopySide w, int64_t inner, int64_t pad, cudaStream_t stream) {
  int lanes = 256;
  while (lanes > 8 && (lanes >= 2 * inner || (lanes > 32 && round_up(inner, lanes) * 7 > inner * 8))) lanes /= 2;
  const int64_t cols = ceil_div(inner, lanes), group = 256 / lanes;
  int64_t blocks = 0;
  for (CopySide* s : {&h, &w}) {
    // no more blocks than occupy the machine four times, unless columns and workers alone are more
    const int64_t row_blocks = std::min(ceil_div(s->rows, group * kCopyRows), std::max<int64_t>(1, 148 * 32 / (cols * s->Z))), n = cols * row_blocks * s->Z;
    if (n > kMaxIndex) return cudaErrorInvalidConfiguration;
    s->row_blocks = (uint32_t)row_blocks;
    s->blocks = (uint32_t)n;
    blocks += n;
  }
  if (blocks > kMaxIndex) return cudaErrorInvalidConfiguration;
  head_copy_kernel<T, D><<<(unsigned)blocks, 256, 0, stream>>>(h, w, inner, pad, lanes, (uint32_t)cols);
  return cudaPeekAtLastError();
}

}  // namespace

extern "C" size_t lsam_head_logprob_workspace_bytes(int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes, int32_t flags) {
  if (!dtype_ok(dtype) || !head_sizes_ok(K, rows, inner, classes)) return 0;
  return head_space(head_plan(dtype, K, rows, inner, classes, (flags & LSAM_HEAD_ALIGNED) != 0), dtype, K, rows, inner, classes, (flags & LSAM_HEAD_SHARED) != 0 || K == 1).total;
}

namespace {

int head_logprob(const Err& err, const void* d_h, const void* d_w, const float* d_bias, int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes,
                 int64_t h_stride_k, int64_t h_stride_row, int64_t w_stride_k, int64_t w_stride_class, int64_t bias_stride_k, const int32_t* d_labels, float* d_logp,
                 float* d_lse, float* d_entropy, void* d_workspace, size_t workspace_bytes, bool starved, void* cuda_stream) {
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (K < 0 || rows < 0 || inner < 1 || classes < 1 || classes > kMaxHead || inner > kMaxHead)
    return err.fail(LSAM_ERR_INVALID, "need K >= 0, rows >= 0, 1 <= inner, classes <= 2^30");
  if (d_logp && !d_labels) return err.fail(LSAM_ERR_INVALID, "d_logp without d_labels");
  if (K == 0 || rows == 0) return LSAM_OK;
  if (K > 65535 || rows > kMaxIndex / K || rows > 4194240) return err.fail(LSAM_ERR_INVALID, "need K <= 65535, rows <= 4194240, K * rows < 2^31");
  if (!strides_ok(K, h_stride_k, rows, h_stride_row, inner, 1) || !strides_ok(K, w_stride_k, classes, w_stride_class, inner, 1) || !strides_ok(K, bias_stride_k, classes, 1, 1, 0))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or a tensor is too large");
  const int64_t total = (int64_t)K * rows, es = (int64_t)dtype_size(dtype);
  const bool shared = w_stride_k == 0 || K == 1;
  const auto aligned16 = [&](const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (n0 == 1 || (s0 > 0 && s0 * es % 16 == 0)) && (n1 == 1 || (s1 > 0 && s1 * es % 16 == 0));
  };
  const bool h_aligned = aligned16(d_h, K, h_stride_k, rows, h_stride_row), w_aligned = aligned16(d_w, shared ? 1 : K, w_stride_k, classes, w_stride_class);
  const HeadPlan plan = head_plan(dtype, K, rows, inner, classes, h_aligned && w_aligned);
  const HeadForm form = plan.form;
  if (starved && form != HEAD_TENSOR) return err.fail(LSAM_ERR_INVALID, "these operands do not go to the tensor cores as they are");
  const HeadSpace sp = head_space(plan, dtype, K, rows, inner, classes, shared);
  if (workspace_bytes < sp.total) return err.fail(LSAM_ERR_WORKSPACE, "workspace smaller than lsam_head_logprob_workspace_bytes()");
  if (reinterpret_cast<uintptr_t>(d_workspace) & 255) return err.fail(LSAM_ERR_WORKSPACE, "workspace not 256-byte aligned");
  PtrCheck pc;
  pc.need(d_h, es); pc.need(d_w, es); pc.need(d_workspace, 256);
  pc.optional(d_bias, 4); pc.optional(d_labels, 4); pc.optional(d_logp, 4); pc.optional(d_lse, 4); pc.optional(d_entropy, 4);
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  char* ws = static_cast<char*>(d_workspace);
  HeadArgs a{rows, inner, classes, total, h_stride_k, h_stride_row, w_stride_k, w_stride_class, bias_stride_k, d_bias, d_labels, 0, 0,
             reinterpret_cast<RowStat*>(ws), reinterpret_cast<float*>(ws + sp.label)};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const T *h = static_cast<const T*>(d_h), *w = static_cast<const T*>(d_w);
    if (form == HEAD_GEMV || form == HEAD_TILES) {
      const SharePlan& p = plan.share;
      a.parts = p.splits;
      a.per_split = p.per_split;
      if (form == HEAD_GEMV) {
        e = launch_gemv<T>(h, w, a, K, w_aligned, stream);
      } else {
        head_score_simt_kernel<T><<<dim3((unsigned)p.splits, (unsigned)ceil_div(rows, kHsM), (unsigned)K), 256, 0, stream>>>(h, w, a);
        e = cudaPeekAtLastError();
      }
      return;
    }
    const HeadTile& q = plan.tile;
    a.parts = 2 * q.runs;
    if (form == HEAD_COPY) {
      using D = typename std::conditional<sizeof(T) == 4, bf16, T>::type;
      constexpr int planes = sizeof(T) == 4 ? 3 : 1;
      D *hc = reinterpret_cast<D*>(ws + sp.h), *wc = reinterpret_cast<D*>(ws + sp.w);
      e = launch_copy<T, D>({h, hc, a.hk, a.hr, rows, K, 0, 0}, {w, wc, a.wk, a.wr, classes, shared ? 1 : K, 0, 0}, inner, sp.pad, stream);
      if (e != cudaSuccess) return;
      a.hr = a.wr = sp.pad;
      a.hk = rows * sp.pad;
      a.wk = classes * sp.pad;
      if (!ht_launch<D>(hc, wc, a, K, q, planes, shared, false, stream, &e)) e = cudaErrorInvalidValue;
    } else if constexpr (sizeof(T) == 2) {
      if (!ht_launch<T>(h, w, a, K, q, 1, shared, starved, stream, &e)) e = cudaErrorInvalidValue;
    }
  });
  if (e == cudaSuccess) {
    // programmatic dependent launch: the join's blocks become resident while the tiles drain and wait for them there
    const ScoreOut out{d_logp, d_lse, d_entropy, nullptr, nullptr, 0, nullptr};
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)ceil_div(total, 8)); cfg.blockDim = dim3(256); cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, head_join_kernel, a, total, out);
  }
  return err.done(e);
}

}  // namespace

extern "C" int lsam_head_logprob(const void* d_h, const void* d_w, const float* d_bias, int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes,
                                 int64_t h_stride_k, int64_t h_stride_row, int64_t w_stride_k, int64_t w_stride_class, int64_t bias_stride_k,
                                 const int32_t* d_labels, float* d_logp, float* d_lse, float* d_entropy, void* d_workspace, size_t workspace_bytes,
                                 void* cuda_stream, char* h_err, size_t h_err_len) {
  return head_logprob(Err("lsam_head_logprob", h_err, h_err_len), d_h, d_w, d_bias, dtype, K, rows, inner, classes, h_stride_k, h_stride_row, w_stride_k, w_stride_class,
                      bias_stride_k, d_labels, d_logp, d_lse, d_entropy, d_workspace, workspace_bytes, false, cuda_stream);
}

extern "C" int lsam_selftest_head_wait(const void* d_h, const void* d_w, int32_t dtype, int32_t K, int64_t rows, int64_t inner, int64_t classes, const int32_t* d_labels,
                                       float* d_logp, float* d_lse, float* d_entropy, void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* h_err,
                                       size_t h_err_len) {
  const bool ok = head_sizes_ok(K, rows, inner, classes);  // sizes that are refused need no strides
  return head_logprob(Err("lsam_selftest_head_wait", h_err, h_err_len), d_h, d_w, nullptr, dtype, K, rows, inner, classes, ok ? rows * inner : 0, inner, ok ? classes * inner : 0, inner, 0,
                      d_labels, d_logp, d_lse, d_entropy, d_workspace, workspace_bytes, true, cuda_stream);
}

namespace {

// Vectors where every row of the three tensors starts on a 16-byte boundary, else single elements.
template <typename T>
cudaError_t launch_dropout(const T* x, const T* skip, T* out, DropArgs a, int32_t K, cudaStream_t stream) {
  const auto aligned = [&](const T* p, int64_t sk, int64_t sr) {
    const int64_t es = sizeof(T);
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && (K == 1 || sk * es % 16 == 0) && (a.rows == 1 || sr * es % 16 == 0));
  };
  if (aligned(x, a.xk, a.xr) && aligned(skip, a.sk, a.sr) && aligned(out, a.ok, a.orr)) {
    const int64_t groups = ceil_div(a.n, 8), total = groups * a.rows * K;
    if (total < kMaxIndex) {
      a.by_groups = FastDiv((uint32_t)groups);
      a.by_rows = FastDiv((uint32_t)a.rows);
      dropout_vec_kernel<T><<<(unsigned)ceil_div(total, 256 * kDropUnroll), 256, 0, stream>>>(x, skip, out, a, (uint32_t)total);
      return cudaPeekAtLastError();
    }
  }
  const int64_t segments = ceil_div(a.n, 256), total = segments * a.rows * K;
  a.by_groups = FastDiv((uint32_t)segments);
  a.by_rows = FastDiv((uint32_t)a.rows);
  dropout_elem_kernel<T><<<(unsigned)ceil_div(total, 8), 256, 0, stream>>>(x, skip, out, a, (uint32_t)total);
  return cudaPeekAtLastError();
}

}  // namespace

extern "C" int lsam_dropout(const void* d_x, const void* d_skip, void* d_out, int32_t dtype, int32_t K, int64_t rows, int64_t n, int64_t x_stride_k,
                            int64_t x_stride_row, int64_t skip_stride_k, int64_t skip_stride_row, int64_t out_stride_k, int64_t out_stride_row, double p,
                            uint64_t seed, uint64_t tick, int32_t layer, int32_t k_offset, void* cuda_stream, char* h_err, size_t h_err_len) {
  const Err err("lsam_dropout", h_err, h_err_len);
  if (!dtype_ok(dtype)) return err.fail(LSAM_ERR_INVALID, "unknown dtype");
  if (!(p >= 0.0 && p <= 1.0)) return err.fail(LSAM_ERR_INVALID, "p outside [0, 1]");
  if (K < 0 || rows < 0 || n < 0) return err.fail(LSAM_ERR_INVALID, "a negative size");
  if (layer < 0 || layer >= LSAM_DROPOUT_LAYERS) return err.fail(LSAM_ERR_INVALID, "layer outside 0 .. LSAM_DROPOUT_LAYERS - 1");
  if (k_offset < 0 || (int64_t)k_offset + K > LSAM_DROPOUT_WORKERS) return err.fail(LSAM_ERR_INVALID, "workers outside 0 .. LSAM_DROPOUT_WORKERS - 1");
  if (K == 0 || rows == 0 || n == 0) return LSAM_OK;
  if (rows > kMaxIndex || n > kMaxIndex) return err.fail(LSAM_ERR_INVALID, "rows and n must be below 2^31");
  if (!strides_ok(K, x_stride_k, rows, x_stride_row, n, 1) || !strides_ok(K, out_stride_k, rows, out_stride_row, n, 1) ||
      (d_skip && !strides_ok(K, skip_stride_k, rows, skip_stride_row, n, 1)))
    return err.fail(LSAM_ERR_INVALID, "a stride is negative or a tensor is too large");
  if (!disjoint(K, out_stride_k, rows, out_stride_row, n, 1)) return err.fail(LSAM_ERR_INVALID, "elements of the output share an address or interleave");
  if ((__int128)ceil_div(n, 256) * rows * K > kMaxIndex) return err.fail(LSAM_ERR_INVALID, "K * rows * ceil(n / 256) must be below 2^31");
  PtrCheck pc;
  pc.need(d_x, dtype_size(dtype)); pc.need(d_out, dtype_size(dtype)); pc.optional(d_skip, dtype_size(dtype));
  if (pc.why) return err.fail(LSAM_ERR_INVALID, pc.why);
  DropArgs a;
  a.rows = rows; a.n = n;
  a.xk = x_stride_k; a.xr = x_stride_row; a.sk = skip_stride_k; a.sr = skip_stride_row; a.ok = out_stride_k; a.orr = out_stride_row;
  a.key0 = (uint32_t)seed ^ 0x64726f70u;  // "drop"
  a.key1 = (uint32_t)(seed >> 32) ^ (uint32_t)(tick >> 32);
  a.tick = (uint32_t)tick;
  a.word2 = ((uint32_t)layer << 20) + (uint32_t)k_offset;
  const uint32_t cut = (uint32_t)std::floor(p * 65536.0 + 0.5);
  a.some = cut < 65536u;
  a.limit = a.some ? cut << 16 : 0u;
  a.scale = a.some ? 65536.f / (float)(65536u - cut) : 0.f;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    e = launch_dropout<T>(static_cast<const T*>(d_x), static_cast<const T*>(d_skip), static_cast<T*>(d_out), a, K, stream);
  });
  return err.done(e);
}
