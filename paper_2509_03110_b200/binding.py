"""Thin ctypes binding of the C ABI in include/lsam.h (argument marshalling only).

PyTorch supplies device memory and the CUDA stream; every step of the method runs in the library's kernels.
There is no CPU fallback: loading fails loudly when the shared library cannot be found or built.
"""
import ctypes as C
import os
import threading
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblsam_b200.so")

LSAM_OK, LSAM_ERR_INVALID, LSAM_ERR_WORKSPACE, LSAM_ERR_STATE, LSAM_ERR_CUDA, LSAM_ERR_NONFINITE, LSAM_ERR_TIMEOUT = range(7)
MODEL_LSQ, MODEL_MLP, MODEL_RESMLP, MODEL_FLAT, MODEL_CNN = 0, 1, 2, 3, 4
GEMM_FP32, GEMM_BF16 = 0, 1
IMPL_AUTO, IMPL_SIMT, IMPL_TCGEN05, IMPL_TCGEN05_1CTA, IMPL_TCGEN05_PAIRS = 0, 1, 2, 3, 4
KERNEL_GAUSSIAN, KERNEL_EXP_POWER, KERNEL_CAUCHY, KERNEL_MATERN32 = 0, 1, 2, 3
FLAG_KEEP_G1, FLAG_STEP_INFO, FLAG_CUDA_GRAPH, FLAG_GRAD_FP32, FLAG_FUSED_UPDATE, FLAG_PDL = 1, 2, 4, 8, 16, 32
PROF_CLASSES = ["schedule", "gather", "gemm_fwd", "gemm_dgrad", "gemm_wgrad", "loss", "bias_grad", "lsq_grad", "norm",
                "perturb", "update", "couple", "copy"]

EXPORTS = [
    "lsam_param_count", "lsam_workspace_bytes", "lsam_init", "lsam_step", "lsam_step_batch", "lsam_stage_batch", "lsam_step_staged", "lsam_couple",
    "lsam_should_couple", "lsam_read_params", "lsam_read_schedule", "lsam_read_step_info", "lsam_read_grads", "lsam_read_grads_replica",
    "lsam_set_external_grads", "lsam_write_state", "lsam_read_state", "lsam_read_counters", "lsam_read_active", "lsam_status",
    "lsam_profile_enable", "lsam_profile_read", "lsam_launch_count", "lsam_uses_tcgen05", "lsam_last_error",
    "lsam_destroy", "lsam_schedule_hash", "lsam_row_norms_static", "lsam_acc_buffer", "lsam_selftest_bounded_wait",
    "lsam_checkpoint_bytes", "lsam_save_checkpoint", "lsam_load_checkpoint", "lsam_read_anchor_gap",
    "lsam_logprob", "lsam_logprob_grad", "lsam_logprob_wide", "lsam_logprob_grad_wide", "lsam_head_logprob", "lsam_head_logprob_workspace_bytes", "lsam_dropout", "lsam_score_batch", "lsam_selftest_head_wait",
]


class LsamConfig(C.Structure):
    _fields_ = [
        ("model", C.c_int32), ("n_layers", C.c_int32), ("widths", C.c_int32 * 9), ("K", C.c_int32), ("batch", C.c_int32),
        ("gemm_dtype", C.c_int32), ("gemm_impl", C.c_int32), ("nesterov", C.c_int32), ("tau", C.c_int32),
        ("stale_max", C.c_int32), ("flags", C.c_int32), ("n_samples", C.c_int64), ("flat_d", C.c_int64),
        ("seed", C.c_uint64), ("mu", C.c_float), ("gamma", C.c_float), ("lam", C.c_float), ("beta", C.c_float),
        ("eta_prime", C.c_float), ("active_num", C.c_int32), ("noise_temp", C.c_float),
        ("K_total", C.c_int32), ("k_offset", C.c_int32), ("kernel_kind", C.c_int32), ("kernel_param", C.c_float), ("dp_average", C.c_int32),
        ("n_conv", C.c_int32), ("img_h", C.c_int32), ("img_w", C.c_int32),
    ]


class LsamError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"lsam error {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load liblsam_b200.so (building it with nvcc if it is absent); raises if neither works."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from . import build as _build

        try:
            _build.build()
        except Exception as e:  # no silent fallback: the CUDA library is the product
            raise RuntimeError(f"liblsam_b200.so is missing and could not be built: {e}") from e
    L = C.CDLL(_LIB_PATH)
    vp, cfgp = C.c_void_p, C.POINTER(LsamConfig)
    L.lsam_param_count.restype = C.c_int64
    L.lsam_param_count.argtypes = [cfgp]
    L.lsam_workspace_bytes.restype = C.c_size_t
    L.lsam_workspace_bytes.argtypes = [cfgp]
    L.lsam_init.argtypes = [C.POINTER(vp), cfgp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.lsam_step.argtypes = [vp, C.c_float, C.c_float]
    L.lsam_step_batch.argtypes = [vp, C.c_float, C.c_float, vp, vp, C.c_int, vp]
    L.lsam_stage_batch.argtypes = [vp, vp, vp, C.c_int]
    L.lsam_step_staged.argtypes = [vp, C.c_float, C.c_float, vp]
    L.lsam_score_batch.argtypes = [vp, vp, vp, C.c_int, C.c_int32, vp, vp, vp, vp, vp]
    L.lsam_couple.argtypes = [vp]
    L.lsam_acc_buffer.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_int64)]
    L.lsam_should_couple.argtypes = [vp]
    L.lsam_read_params.argtypes = [vp, C.c_int, vp, C.c_int64, C.c_int]
    L.lsam_read_schedule.argtypes = [vp, C.c_int64, vp, vp, vp]
    L.lsam_read_step_info.argtypes = [vp, vp, vp, vp]
    L.lsam_read_grads.argtypes = [vp, C.c_int, vp]
    L.lsam_read_grads_replica.argtypes = [vp, C.c_int, C.c_int, vp]
    L.lsam_set_external_grads.argtypes = [vp, vp, vp]
    L.lsam_write_state.argtypes = [vp, vp, vp, vp]
    L.lsam_read_state.argtypes = [vp, vp, vp, vp]
    L.lsam_read_counters.argtypes = [vp, vp, vp, vp]
    L.lsam_read_active.argtypes = [vp, vp]
    L.lsam_status.argtypes = [vp]
    L.lsam_read_anchor_gap.argtypes = [vp, vp]
    L.lsam_checkpoint_bytes.restype = C.c_size_t
    L.lsam_checkpoint_bytes.argtypes = [vp]
    L.lsam_save_checkpoint.argtypes = [vp, vp, C.c_size_t]
    L.lsam_load_checkpoint.argtypes = [vp, vp, C.c_size_t]
    L.lsam_selftest_bounded_wait.argtypes = [vp, C.c_uint32]
    L.lsam_profile_enable.argtypes = [vp, C.c_int]
    L.lsam_profile_read.argtypes = [vp, vp, vp]
    L.lsam_launch_count.restype = C.c_int64
    L.lsam_launch_count.argtypes = [vp]
    L.lsam_uses_tcgen05.argtypes = [vp]
    L.lsam_last_error.restype = C.c_char_p
    L.lsam_last_error.argtypes = [vp]
    L.lsam_destroy.restype = None
    L.lsam_destroy.argtypes = [vp]
    L.lsam_schedule_hash.restype = C.c_uint64
    L.lsam_schedule_hash.argtypes = [C.c_uint64, C.c_int, C.c_uint64, C.c_uint64, C.c_uint64]
    L.lsam_row_norms_static.argtypes = [vp, C.c_int64, C.c_int64, C.c_int32, vp, vp, C.c_char_p, C.c_size_t]
    i32, i64, err = C.c_int32, C.c_int64, [vp, C.c_char_p, C.c_size_t]  # err: stream and error buffer
    L.lsam_logprob.argtypes = [vp, i32, i32] + [i64] * 5 + [vp, i32] + [vp] * 5 + err
    L.lsam_logprob_grad.argtypes = [vp, i32, i32] + [i64] * 5 + [vp] * 6 + [i64] * 3 + err
    L.lsam_logprob_wide.argtypes = [vp, i32, i32] + [i64] * 5 + [vp, i32] + [vp] * 6 + err
    L.lsam_logprob_grad_wide.argtypes = [vp, i32, i32] + [i64] * 5 + [vp] * 7 + [i64] * 3 + err
    L.lsam_head_logprob_workspace_bytes.restype = C.c_size_t
    L.lsam_head_logprob_workspace_bytes.argtypes = [i32, i32, i64, i64, i64, i32]
    L.lsam_head_logprob.argtypes = [vp, vp, vp, i32, i32] + [i64] * 8 + [vp] * 5 + [C.c_size_t] + err
    L.lsam_selftest_head_wait.argtypes = [vp, vp, i32, i32] + [i64] * 3 + [vp] * 5 + [C.c_size_t] + err
    L.lsam_dropout.argtypes = [vp, vp, vp, i32, i32] + [i64] * 8 + [C.c_double, C.c_uint64, C.c_uint64, i32, i32] + err
    _lib = L
    return L


def make_config(model, widths=(), K=1, batch=1, gemm_dtype=GEMM_FP32, gemm_impl=IMPL_AUTO, mu=0.9, nesterov=1,
                gamma=1e-12, lam=0.0, tau=4, beta=0.9, eta_prime=1.0, stale_max=0, seed=0, n_samples=1, flat_d=0, flags=0,
                active_num=256, noise_temp=0.0, K_total=0, k_offset=0, kernel_kind=KERNEL_GAUSSIAN, kernel_param=0.0, dp_average=0, n_conv=0, img_h=0, img_w=0):
    c = LsamConfig()
    c.model = model
    widths = list(widths)
    c.n_layers = max(len(widths) - 1, 0) if model in (MODEL_MLP, MODEL_RESMLP, MODEL_CNN) else (1 if model == MODEL_LSQ else 0)
    for i, w in enumerate(widths):
        c.widths[i] = int(w)
    c.K, c.batch, c.gemm_dtype, c.gemm_impl, c.nesterov, c.tau = int(K), int(batch), int(gemm_dtype), int(gemm_impl), int(nesterov), int(tau)
    c.stale_max, c.flags, c.n_samples, c.flat_d, c.seed = int(stale_max), int(flags), int(n_samples), int(flat_d), int(seed)
    c.mu, c.gamma, c.lam, c.beta, c.eta_prime = mu, gamma, lam, beta, eta_prime
    c.active_num = int(active_num)
    c.noise_temp = noise_temp
    c.K_total, c.k_offset = int(K_total), int(k_offset)
    c.kernel_kind, c.kernel_param, c.dp_average = int(kernel_kind), kernel_param, int(dp_average)
    c.n_conv, c.img_h, c.img_w = int(n_conv), int(img_h), int(img_w)
    return c


def lsam_param_count(cfg):
    return int(lib().lsam_param_count(C.byref(cfg)))


def lsam_workspace_bytes(cfg):
    return int(lib().lsam_workspace_bytes(C.byref(cfg)))


def lsam_schedule_hash(seed, tag, t, k, j):
    return int(lib().lsam_schedule_hash(seed, tag, t, k, j))


STATIC_NORM_MAX_PARTIALS = 262144


def lsam_row_norms_static(g, n, out, stream=None):
    """Row norms of the CUDA tensor g [K, ld] (first n columns) into the CUDA tensor out [K], with no allocation.

    For callers that may not allocate device memory (see include/lsam.h): the partial sums live in an array inside
    the library.  Returns (status, message).  Calls that overlap on one GPU race on that array; the first call on a
    device should be made outside stream capture.
    """
    K, ld = g.shape
    err = C.create_string_buffer(256)
    s = C.c_void_p(stream.cuda_stream) if stream is not None else None
    rc = lib().lsam_row_norms_static(C.c_void_p(g.data_ptr()), ld, int(n), K, C.c_void_p(out.data_ptr()), s, err, 256)
    return int(rc), err.value.decode()


# ---- operators around a classifier's head (include/lsam.h, last section)
# Plain calls on tensors: autograd records none of them and does not see what is written through `out`.
FP32, BF16, FP16 = 0, 1, 2
HEAD_ALIGNED, HEAD_SHARED = 1, 2
TOP_MAX, DROPOUT_LAYERS, DROPOUT_WORKERS = 32, 4096, 1 << 20


class _Scores(NamedTuple):
    logp: object
    lse: object
    entropy: object
    top_logp: object
    top_idx: object


class LogProb(_Scores):
    """Scores of rows of logits: fp32 [..., rows] (top_logp and int32 top_idx: [..., rows, top_k]); None where not asked for.

    lse_low, beside the tuple: what the rounding of lse to 32 bits leaves out (lsam_logprob only, else None)."""

    lse_low = None


def _invalid(msg):
    return LsamError(LSAM_ERR_INVALID, msg)


# Host time is what bounds the smallest calls (an allocation through torch.empty with keywords is 2 to 3 us, a stream object 2 us), so the
# operators allocate through an empty tensor of the right type and device, and ask for the stream's handle alone.
_torch = _raw_stream = None
_codes = {}  # torch dtype -> LSAM_FP32 / LSAM_BF16 / LSAM_FP16
_protos = {}  # device -> empty float32 tensor: what results are allocated like; it holds no memory
_err = threading.local()  # one message buffer per thread


def _load():
    """torch, imported with the first operator call."""
    global _torch, _raw_stream
    if _torch is None:
        import torch

        _codes.update({torch.float32: FP32, torch.bfloat16: BF16, torch.float16: FP16})
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream = (lambda dev: raw(dev.index)) if raw is not None else (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        _torch = torch
    return _torch


def _proto(dev):
    p = _protos.get(dev)
    if p is None:
        p = _protos[dev] = _torch.empty(0, dtype=_torch.float32, device=dev)
    return p


def _call(fn, *args):
    try:
        buf = _err.buf
    except AttributeError:
        buf = _err.buf = C.create_string_buffer(256)
    rc = fn(*args, buf, 256)
    if rc != LSAM_OK:
        raise LsamError(rc, buf.value.decode())


def _stacked(t, what):
    """K, rows, columns and the strides of a [rows, columns] or [K, rows, columns] tensor."""
    n = t.dim()
    if n == 3:
        if t.shape[0] >> 31:
            raise _invalid(f"{what}: 2^31 workers or more")
        return (*t.shape, *t.stride())
    if n == 2:
        return (1, *t.shape, 0, *t.stride())
    raise _invalid(f"{what} must have 2 or 3 dimensions")


def _code(t, what):
    code = _codes.get(t.dtype)
    if code is None:
        raise _invalid(f"{what}: {t.dtype} is not one of float32, bfloat16, float16")
    if not t.is_cuda:
        raise _invalid("the operators take CUDA tensors: there is no CPU path")
    return code


def _ptr(t, what, shape, dtype, dev):
    """Address of a dense per-row array, None if it is not given."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise _invalid(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")
    return t.data_ptr()


def _on(stream, fn, *tensors):
    """Runs an operator with `stream` as the current stream, so that what it allocates belongs to that stream.  The memory of `tensors`, what the
    caller handed in, is not handed out again before `stream` has passed the call, even if the caller drops them at once."""
    with _torch.cuda.stream(stream):
        r = fn()
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return r


def lsam_logprob(logits, labels=None, top_k=0, stream=None):
    """Log probability of the label, log-sum-exp, entropy and the top_k alternatives of every row of logits.

    logits: [rows, classes] or [K, rows, classes], float32 / bfloat16 / float16, any strides (a context's own logits have the sample
    index contiguous: a transposed view).  labels: int32 [rows] / [K, rows]; negative = the row is left out (zeros, index -1), None = no
    logp.  The rules for masks, NaN and ties stand in include/lsam.h.  Returns LogProb.
    stream: None = the current one.  Another one has to be ordered behind what produced the inputs; the results belong to it, so a stream that reads
    them has to be ordered behind it in turn.  (The same for the other operators.)
    """
    torch = _load()
    if stream is not None:
        return _on(stream, lambda: lsam_logprob(logits, labels, top_k), logits, labels)
    K, R, V, sk, sr, sc = _stacked(logits, "logits")
    code = _code(logits, "logits")
    dev = logits.device
    lead = (K, R) if logits.dim() == 3 else (R,)
    pl = None if labels is None else _ptr(labels, "labels", lead, torch.int32, dev)
    n = 4 * K * R  # bytes of a per-row result
    buf = _proto(dev).new_empty((3 if labels is None else 4, *lead))
    if labels is None:
        logp = pp = None
        lse, ent, low = buf.unbind(0)
        p = buf.data_ptr()
    else:
        logp, lse, ent, low = buf.unbind(0)
        pp = buf.data_ptr()
        p = pp + n
    tv = ti = pv = pi = None
    if top_k:
        if not 0 < top_k <= TOP_MAX:
            raise _invalid(f"top_k outside 0 .. {TOP_MAX}")
        buf = buf.new_empty((2, *lead, top_k))
        tv, ti = buf.unbind(0)
        ti = ti.view(torch.int32)
        pv = buf.data_ptr()
        pi = pv + n * top_k
    _call(lib().lsam_logprob_wide, logits.data_ptr(), code, K, R, V, sk, sr, sc, pl, top_k, pp, p, p + 2 * n, p + n, pv, pi, _raw_stream(dev))
    r = tuple.__new__(LogProb, (logp, lse, ent, tv, ti))  # without the check of a named tuple's arguments
    r.lse_low = low
    return r


def lsam_logprob_grad(logits, labels, lse, dlogp, entropy=None, dentropy=None, out=None, stream=None, lse_low=None):
    """Gradient with respect to the logits of a loss whose derivatives by logp and entropy are dlogp and dentropy (either may be None).

    lse: what lsam_logprob returned for these logits, whole (then entropy and lse_low are taken from it where they are not given), or its lse alone, with
    which the probabilities of a row are off by a factor of 1 +- |lse| 2^-24.  out: tensor of the logits' shape and type to write (logits itself is
    allowed), None = a new one.  Returns it.
    """
    torch = _load()
    if isinstance(lse, LogProb):
        if lse_low is None:
            lse_low = lse.lse_low
        if entropy is None and dentropy is not None:
            entropy = lse.entropy
        lse = lse.lse
    if stream is not None:
        return _on(stream, lambda: lsam_logprob_grad(logits, labels, lse, dlogp, entropy, dentropy, out, None, lse_low), logits, labels, lse, dlogp, entropy, dentropy, out, lse_low)
    K, R, V, sk, sr, sc = _stacked(logits, "logits")
    code = _code(logits, "logits")
    dev = logits.device
    lead = logits.shape[:-1]
    f32 = torch.float32
    pl = _ptr(labels, "labels", lead, torch.int32, dev)
    ps = _ptr(lse, "lse", lead, f32, dev)
    if ps is None:
        raise _invalid("lse is needed")
    pw, pe, pa, pb = _ptr(lse_low, "lse_low", lead, f32, dev), _ptr(entropy, "entropy", lead, f32, dev), _ptr(dlogp, "dlogp", lead, f32, dev), _ptr(dentropy, "dentropy", lead, f32, dev)
    if out is None:
        out = torch.empty_like(logits)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != dev:
        raise _invalid("out must have the shape, type and device of logits")
    ok, orow, oc = _stacked(out, "out")[3:]
    _call(lib().lsam_logprob_grad_wide, logits.data_ptr(), code, K, R, V, sk, sr, sc, pl, ps, pw, pe, pa, pb, out.data_ptr(), ok, orow, oc, _raw_stream(dev))
    return out


def lsam_head_logprob(h, w, labels=None, bias=None, stream=None):
    """lsam_logprob's first three results for the logits h w^T + bias, without storing them.

    h: [rows, inner] or [K, rows, inner]; w: [classes, inner] (shared by the workers) or [K, classes, inner]; bias: fp32 [classes] /
    [K, classes]; the inner index contiguous.  Returns LogProb without alternatives.
    """
    torch = _load()
    if stream is not None:
        return _on(stream, lambda: lsam_head_logprob(h, w, labels, bias), h, w, labels, bias)
    K, R, D, hk, hr, hc = _stacked(h, "h")
    KW, V, DW, wk, wc, wi = _stacked(w, "w")
    code = _code(h, "h")
    dev = h.device
    lead = h.shape[:-1]
    if DW != D or w.dtype != h.dtype or w.device != dev or (w.dim() == 3 and KW != K):
        raise _invalid("w must be [classes, inner] or [K, classes, inner] of the type and device of h")
    if (hc != 1 or wi != 1) and D > 1:
        raise _invalid("the inner index of h and w must be contiguous")
    pl = _ptr(labels, "labels", lead, torch.int32, dev)
    pb, bk = None, 0
    if bias is not None:
        pb = _ptr(bias, "bias", (V,) if bias.dim() == 1 else (K, V), torch.float32, dev)
        bk = V if bias.dim() == 2 else 0
    f32 = _proto(dev)
    if labels is None:
        logp = None
        lse, ent = f32.new_empty((2, *lead)).unbind(0)
    else:
        logp, lse, ent = f32.new_empty((3, *lead)).unbind(0)
    L = lib()
    ph, pw = h.data_ptr(), w.data_ptr()
    unit = 3 if code == FP32 else 7  # elements of 16 bytes, minus one
    aligned = not ((ph | pw) & 15) and not ((hk if K > 1 else 0) | (hr if R > 1 else 0) | (wk if K > 1 else 0) | (wc if V > 1 else 0)) & unit and (hr > 0 or R == 1) and (hk > 0 or K == 1) and (wc > 0 or V == 1)
    nbytes = L.lsam_head_logprob_workspace_bytes(code, K, R, D, V, (HEAD_ALIGNED if aligned else 0) | (0 if wk else HEAD_SHARED)) if K and R else 0
    ws = f32.new_empty(nbytes // 4 + 64)
    _call(L.lsam_head_logprob, ph, pw, pb, code, K, R, D, V, hk, hr, wk, wc, bk, pl, None if logp is None else logp.data_ptr(), lse.data_ptr(),
          ent.data_ptr(), (ws.data_ptr() + 255) // 256 * 256, nbytes, _raw_stream(dev))
    return LogProb(logp, lse, ent, None, None)


def lsam_dropout(x, p, seed, tick, layer=0, k_offset=0, skip=None, out=None, stream=None):
    """skip + dropout(x) with a mask that is a function of (seed, tick, layer, worker, row, column) and is never stored.

    x: [rows, n] or [K, rows, n], float32 / bfloat16 / float16, columns contiguous; worker k_offset + k owns x[k].  The backward pass is the
    same call on the gradient, without skip.  out: tensor to write (x or skip itself is allowed), None = a new one.  Returns it.
    """
    torch = _load()
    if stream is not None:
        return _on(stream, lambda: lsam_dropout(x, p, seed, tick, layer, k_offset, skip, out), x, skip, out)
    K, R, n, xk, xr, xc = _stacked(x, "x")
    code = _code(x, "x")
    dev = x.device
    if not 0 <= seed < 1 << 64 or not 0 <= tick < 1 << 64:
        raise _invalid("seed and tick are unsigned 64-bit numbers")
    if not 0 <= layer < DROPOUT_LAYERS or not 0 <= k_offset < DROPOUT_WORKERS:
        raise _invalid(f"layer outside 0 .. {DROPOUT_LAYERS - 1} or k_offset outside 0 .. {DROPOUT_WORKERS - 1}")
    if out is None:
        out = x.new_empty(x.shape)
    elif out.shape != x.shape or out.dtype != x.dtype or out.device != dev:
        raise _invalid("out must have the shape, type and device of x")
    ok, orow, oc = _stacked(out, "out")[3:]
    ps, sk, sr, sc = None, 0, 0, 1
    if skip is not None:
        if skip.shape != x.shape or skip.dtype != x.dtype or skip.device != dev:
            raise _invalid("skip must have the shape, type and device of x")
        ps = skip.data_ptr()
        sk, sr, sc = _stacked(skip, "skip")[3:]
    if (xc != 1 or oc != 1 or sc != 1) and n > 1:
        raise _invalid("the columns of x, skip and out must be contiguous")
    _call(lib().lsam_dropout, x.data_ptr(), ps, out.data_ptr(), code, K, R, n, xk, xr, sk, sr, ok, orow, p, seed, tick, layer, k_offset,
          _raw_stream(dev))
    return out


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dev_ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


class Lsam:
    """One LSAM context on the current CUDA device.  Tensors passed in are torch CUDA tensors (fp32 / int32)."""

    def __init__(self, cfg, X=None, Y=None, x0=None, y0=None, stream=None):
        import torch

        self._torch = torch
        self.cfg = cfg
        self.K = cfg.K
        self.d = lsam_param_count(cfg)
        if self.d <= 0:
            raise LsamError(LSAM_ERR_INVALID, "invalid configuration")
        nbytes = lsam_workspace_bytes(cfg)
        dev = x0.device
        assert dev.type == "cuda", "x0 must be a CUDA tensor: there is no CPU path"
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)
        self._keep = [X, Y]
        x0 = x0.contiguous().float()
        y0 = y0.contiguous().float()
        assert x0.numel() == self.K * self.d and y0.numel() == self.d
        h = C.c_void_p()
        rc = lib().lsam_init(C.byref(h), C.byref(cfg), _dev_ptr(X), _dev_ptr(Y), _dev_ptr(x0), _dev_ptr(y0),
                             C.c_void_p(self._ws_ptr), nbytes, C.c_void_p(self.stream.cuda_stream))
        if rc != LSAM_OK:
            raise LsamError(rc, "lsam_init failed")
        self._h = h
        self.stream.synchronize()  # x0 / y0 may be temporaries

    # -- lifetime
    def close(self):
        if getattr(self, "_h", None):
            self.stream.synchronize()
            lib().lsam_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != LSAM_OK:
            raise LsamError(rc, lib().lsam_last_error(self._h).decode())

    # -- the four calls of the method
    def step(self, eta, rho):
        self._check(lib().lsam_step(self._h, eta, rho))

    def step_batch(self, eta, rho, xb, yb, h_loss=None):
        """xb / yb: pinned host tensors or numpy arrays (on_host) or CUDA tensors; h_loss: numpy float32 [K] or None."""
        torch = self._torch
        on_host = not (isinstance(xb, torch.Tensor) and xb.is_cuda)
        px = C.c_void_p(xb.data_ptr()) if isinstance(xb, torch.Tensor) else _np_ptr(xb)
        py = C.c_void_p(yb.data_ptr()) if isinstance(yb, torch.Tensor) else _np_ptr(yb)
        self._check(lib().lsam_step_batch(self._h, eta, rho, px, py, 1 if on_host else 0, _np_ptr(h_loss)))

    def stage_batch(self, xb, yb):
        """Prefetch a minibatch (pinned host tensors / numpy arrays, or CUDA tensors) into the next staging slot."""
        torch = self._torch
        on_host = not (isinstance(xb, torch.Tensor) and xb.is_cuda)
        px = C.c_void_p(xb.data_ptr()) if isinstance(xb, torch.Tensor) else _np_ptr(xb)
        py = C.c_void_p(yb.data_ptr()) if isinstance(yb, torch.Tensor) else _np_ptr(yb)
        self._check(lib().lsam_stage_batch(self._h, px, py, 1 if on_host else 0))

    def step_staged(self, eta, rho, h_loss=None):
        self._check(lib().lsam_step_staged(self._h, eta, rho, _np_ptr(h_loss)))

    def score_batch(self, xb, yb=None, top_k=0):
        """Log probability of the labels, log-sum-exp, entropy and top_k alternatives of a minibatch under every worker's iterate.

        xb [K, B, in] float32, yb [K, B] int32 or None: both CUDA tensors, or both host tensors / numpy arrays (pinned ones are read when the context's
        stream gets there: they must stay as they are, and be kept, until it has passed the call).  Returns LogProb of CUDA tensors [K, B].
        Runs on the context's stream: other streams order their reads of the result behind it, and it behind what produced xb and yb.
        """
        torch = _load()
        if not 0 <= top_k <= TOP_MAX:
            raise _invalid(f"top_k outside 0 .. {TOP_MAX}")
        K, B = self.K, self.cfg.batch
        on_host = not (isinstance(xb, torch.Tensor) and xb.is_cuda)
        for t, what, ty, shape in ((xb, "xb", "float32", None), (yb, "yb", "int32", (K, B))):
            if t is None:
                continue
            ok = str(t.dtype).replace("torch.", "") == ty and (t.is_contiguous() if isinstance(t, torch.Tensor) else t.flags.c_contiguous)
            if not ok or tuple(t.shape[:2]) != (K, B) or (shape and tuple(t.shape) != shape) or on_host == (isinstance(t, torch.Tensor) and t.is_cuda):
                raise _invalid(f"{what} must be a contiguous {ty} array [K, B, ...] on the {'host' if on_host else 'device'}")
        n_in = self.cfg.widths[0] * (self.cfg.img_h * self.cfg.img_w if self.cfg.model == MODEL_CNN else 1)
        if int(np.prod(tuple(xb.shape[2:]))) != n_in:
            raise _invalid(f"a row of xb must hold {n_in} features")
        with torch.cuda.stream(self.stream):
            f32 = _proto(self.workspace.device)
            logp, lse, ent = f32.new_empty((3, K, B)).unbind(0)
            tv, ti = f32.new_empty((2, K, B, top_k)).unbind(0) if top_k else (None, None)
            logp, ti = None if yb is None else logp, None if ti is None else ti.view(torch.int32)
        ptr = lambda a: None if a is None else C.c_void_p(a.data_ptr()) if isinstance(a, torch.Tensor) else _np_ptr(a)  # noqa: E731
        self._check(lib().lsam_score_batch(self._h, ptr(xb), ptr(yb), 1 if on_host else 0, top_k, ptr(logp), ptr(lse), ptr(ent), ptr(tv), ptr(ti)))
        if not on_host:  # their memory is not handed out again before the context's stream has read it
            for t in (xb, yb):
                if t is not None:
                    t.record_stream(self.stream)
        return LogProb(logp, lse, ent, tv, ti)

    def should_couple(self):
        return bool(lib().lsam_should_couple(self._h))

    def couple(self):
        return int(lib().lsam_couple(self._h))

    def acc_tensor(self):
        """The iterate accumulator as a CUDA fp32 tensor that aliases the workspace (sharded runs all-reduce it in place)."""
        p, n = C.c_void_p(), C.c_int64()
        self._check(lib().lsam_acc_buffer(self._h, C.byref(p), C.byref(n)))
        off = int(p.value) - self.workspace.data_ptr()
        return self.workspace[off:off + 4 * int(n.value)].view(self._torch.float32)

    def read_params(self, which, out=None):
        """Returns a numpy fp32 [d] (host copy) or fills the CUDA tensor `out`."""
        if out is not None:
            self._check(lib().lsam_read_params(self._h, int(which), _dev_ptr(out), out.numel(), 1))
            return out
        dst = np.empty(self.d, dtype=np.float32)
        self._check(lib().lsam_read_params(self._h, int(which), _np_ptr(dst), self.d, 0))
        return dst

    # -- helpers
    def read_all_params(self):
        return np.stack([self.read_params(k) for k in range(self.K)])

    def read_schedule(self, t, want_ver=True):
        K, B = self.K, max(self.cfg.batch, 1)
        idx = np.zeros((K, B), dtype=np.int32)
        stale = np.zeros(K, dtype=np.int32)
        ver = np.zeros(K, dtype=np.int32)
        self._check(lib().lsam_read_schedule(self._h, int(t), _np_ptr(idx), _np_ptr(stale), _np_ptr(ver) if want_ver else None))
        return idx, stale, ver

    def read_step_info(self):
        loss, n1, n2 = (np.zeros(self.K, dtype=np.float32) for _ in range(3))
        self._check(lib().lsam_read_step_info(self._h, _np_ptr(loss), _np_ptr(n1), _np_ptr(n2)))
        return loss, n1, n2

    def read_anchor_gap(self):
        """||x_k - y|| for every worker against the current centre (numpy fp32 [K])."""
        out = np.zeros(self.K, dtype=np.float32)
        self._check(lib().lsam_read_anchor_gap(self._h, _np_ptr(out)))
        return out

    def read_grads(self, which_pass):
        out = np.empty((self.K, self.d), dtype=np.float32)
        self._check(lib().lsam_read_grads(self._h, int(which_pass), _np_ptr(out)))
        return out

    def read_grads_replica(self, which_pass, k):
        out = np.empty(self.d, dtype=np.float32)
        self._check(lib().lsam_read_grads_replica(self._h, int(which_pass), int(k), _np_ptr(out)))
        return out

    def set_external_grads(self, g1, g2):
        self._keep += [g1, g2]
        self._check(lib().lsam_set_external_grads(self._h, _dev_ptr(g1), _dev_ptr(g2)))

    def write_state(self, x=None, v=None, y=None):
        cv = lambda a: None if a is None else a.contiguous().float()
        x, v, y = cv(x), cv(v), cv(y)
        self._check(lib().lsam_write_state(self._h, _dev_ptr(x), _dev_ptr(v), _dev_ptr(y)))
        self.stream.synchronize()

    def read_state(self):
        v = np.empty((self.K, self.d), dtype=np.float32)
        acc = np.empty(self.d, dtype=np.float32)
        gprev = np.empty(self.d, dtype=np.float32)
        self._check(lib().lsam_read_state(self._h, _np_ptr(v), _np_ptr(acc), _np_ptr(gprev)))
        return dict(v=v, acc=acc, gprev=gprev)

    def read_active(self):
        a = np.zeros(self.K, dtype=np.int32)
        self._check(lib().lsam_read_active(self._h, _np_ptr(a)))
        return a

    def counters(self):
        t = np.zeros(1, dtype=np.int64)
        ty = np.zeros(1, dtype=np.int64)
        tx = np.zeros(self.K, dtype=np.int64)
        self._check(lib().lsam_read_counters(self._h, _np_ptr(t), _np_ptr(ty), _np_ptr(tx)))
        return int(t[0]), int(ty[0]), tx

    def status(self):
        return int(lib().lsam_status(self._h))

    def last_error(self):
        return (lib().lsam_last_error(self._h) or b"").decode()

    def save_checkpoint(self):
        """The whole state of the run as a numpy byte array (host)."""
        n = int(lib().lsam_checkpoint_bytes(self._h))
        buf = np.empty(n, dtype=np.uint8)
        self._check(lib().lsam_save_checkpoint(self._h, _np_ptr(buf), n))
        return buf

    def load_checkpoint(self, buf):
        buf = np.ascontiguousarray(buf, dtype=np.uint8)
        self._check(lib().lsam_load_checkpoint(self._h, _np_ptr(buf), buf.size))

    def selftest_bounded_wait(self, polls=2048):
        """Enqueue a wait that is bound to expire (see include/lsam.h); status() then reports LSAM_ERR_TIMEOUT."""
        self._check(lib().lsam_selftest_bounded_wait(self._h, int(polls)))

    def profile_enable(self, on=True):
        self._check(lib().lsam_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        ms = np.zeros(len(PROF_CLASSES), dtype=np.float64)
        n = np.zeros(len(PROF_CLASSES), dtype=np.int64)
        self._check(lib().lsam_profile_read(self._h, _np_ptr(ms), _np_ptr(n)))
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(PROF_CLASSES)}

    def launch_count(self):
        return int(lib().lsam_launch_count(self._h))

    def uses_tcgen05(self):
        return bool(lib().lsam_uses_tcgen05(self._h))
