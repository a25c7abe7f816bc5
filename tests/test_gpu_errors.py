"""A call that fails is reported by that call alone."""
import ctypes as C
import os

import pytest
import torch

from paper_2509_03110_b200 import binding as G
from test_gpu_score_batch import CONFIGS, make

pytestmark = pytest.mark.gpu


def runtime():
    """The CUDA runtime that torch has loaded."""
    for line in open("/proc/self/maps"):
        path = line.split()[-1]
        if os.path.basename(path).startswith("libcudart.so"):
            return C.CDLL(path)
    pytest.skip("no shared CUDA runtime in this process")


def test_a_failed_call_leaves_no_error_for_the_next():
    rt = runtime()
    ctx, xb, yb, classes = make(CONFIGS["mlp_fp32"])
    ctx.step(0.02, 0.05)
    r = ctx.score_batch(xb, yb)
    logits = torch.randn((1, 40, 100), device="cuda")
    labels = torch.zeros((1, 40), device="cuda", dtype=torch.int32)
    want = G.lsam_logprob(logits, labels)
    other, oxb, oyb, _ = make(CONFIGS["mlp_fp32"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    # reading the status waits for the stream, which a stream that is being captured does not allow: an error on the host, nothing runs
    cfg = G.make_config(G.MODEL_FLAT, K=2, flat_d=64)
    ctx2 = G.Lsam(cfg, None, None, torch.zeros(2, 64, device="cuda"), torch.zeros(64, device="cuda"), stream=side)
    torch.cuda.synchronize()
    graph = C.c_void_p()
    assert rt.cudaStreamBeginCapture(C.c_void_p(side.cuda_stream), 1) == 0  # 1: this thread's calls on this stream
    rc = ctx2.status()
    assert rt.cudaStreamEndCapture(C.c_void_p(side.cuda_stream), C.byref(graph)) != 0  # the capture was broken off
    rt.cudaGetLastError()
    assert rc == G.LSAM_ERR_CUDA
    # what follows has nothing to do with it
    got = G.lsam_logprob(logits, labels)
    assert torch.equal(got.lse, want.lse)
    again = ctx.score_batch(xb, yb)
    assert torch.equal(again.lse, r.lse)
    assert ctx2.status() == G.LSAM_OK
    other.step_batch(0.02, 0.05, oxb, oyb)
    assert other.status() == G.LSAM_OK
    for c in (ctx, ctx2, other):
        c.close()
