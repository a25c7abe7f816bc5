"""A head call whose copies never arrive: its waits run out, the call ends, and every row says so."""
import ctypes as C

import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu


# one CTA with few rows, one with a full tile of rows, pairs, pairs with several units of work each, several workers
@pytest.mark.parametrize("K, rows, D, V", [(1, 4, 256, 5000), (1, 128, 64, 300), (1, 200, 1024, 3000), (1, 700, 128, 40000), (3, 257, 136, 1000)])
@pytest.mark.parametrize("stale", [float("-inf"), -3e38, 0.0, 7.0])
def test_rows_whose_waits_run_out_are_nan(K, rows, D, V, stale):
    g = torch.Generator(device="cuda").manual_seed(V)
    h = torch.randn((K, rows, D), generator=g, device="cuda").bfloat16()
    w = torch.randn((K, V, D), generator=g, device="cuda").bfloat16() / 16
    y = torch.randint(0, V, (K, rows), generator=g, device="cuda", dtype=torch.int32)
    y[0, 0], y[K - 1, rows - 1] = -1, V
    nbytes = G.lib().lsam_head_logprob_workspace_bytes(G.BF16, K, rows, D, V, G.HEAD_ALIGNED)
    ws = torch.full((nbytes // 4 + 64,), stale, device="cuda")  # what an earlier call may have left where the labels' logits go
    out = torch.zeros((3, K, rows), device="cuda")
    torch.cuda.synchronize()
    err = C.create_string_buffer(256)
    rc = G.lib().lsam_selftest_head_wait(h.data_ptr(), w.data_ptr(), G.BF16, K, rows, D, V, y.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
                                         (ws.data_ptr() + 255) // 256 * 256, nbytes, torch.cuda.current_stream().cuda_stream, err, 256)
    assert rc == G.LSAM_OK, err.value
    torch.cuda.synchronize()
    left = (y < 0).expand(3, K, rows)
    assert (out[left] == 0).all() and torch.isnan(out[~left]).all()
    r = G.lsam_head_logprob(h, w, y)  # and the next call is as ever
    assert torch.isfinite(r.lse).all() and torch.isfinite(r.entropy).all() and torch.isnan(r.logp[K - 1, rows - 1])


def test_the_self_test_wants_the_tensor_core_form():
    h, y = torch.zeros((4, 64), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ws, err = torch.zeros(1 << 20, device="cuda"), C.create_string_buffer(256)
    rc = G.lib().lsam_selftest_head_wait(h.data_ptr(), h.data_ptr(), G.FP32, 1, 4, 64, 4, y.data_ptr(), None, h.data_ptr(), None, (ws.data_ptr() + 255) // 256 * 256, 1 << 21, None, err, 256)
    assert rc == G.LSAM_ERR_INVALID and b"tensor cores" in err.value
