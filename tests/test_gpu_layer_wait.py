"""Waits of the operators for layers and updates that run out: what they concern is NaN, nothing is finite and wrong, and the next call is as ever."""
import ctypes as C

import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu
SMS = 148


def scratch(nbytes):
    ws = torch.full((nbytes // 4 + 64,), 3.0, device="cuda")
    return ws, (ws.data_ptr() + 255) // 256 * 256


# two, four and eight blocks a cluster, rows with and without vectors; every block has at least four rows, one three of them at the end
@pytest.mark.parametrize("rows, n", [(74 * 5 - 2, 5000), (74 * 4, 5003), (37 * 7, 12000), (18 * 5, 20000), (18 * 6 - 3, 32767)])
def test_sums_of_a_cluster_that_never_arrive(rows, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, b, dy, du = (rand(rows, n) for _ in range(4))
    z, pw, nw = rand(rows, 1), 1 + 0.1 * rand(n), 1 + 0.1 * rand(n)
    how = dict(branch=b, gate=z, post_weight=pw, pre_weight=nw)
    inv = lambda t: (t.double().pow(2).mean(-1) + 1e-6).rsqrt().float()  # noqa: E731
    fwd = G.ResidualNorm(x, None, inv(b), inv(x))
    want = G.lsam_residual_norm_grad(fwd, dy, du, act="sigmoid", **how)
    got = [torch.full_like(t, 5.0) for t in want]  # dx, dbranch, dgate, the weights'
    row = lambda t: G.LsamRows(t.data_ptr(), 0, n)  # noqa: E731
    r = G.LsamResidual(G.FP32, 1, rows, n, 1, 1, G.GATE_ROW, 1, 1.0, 1.0, 1.0, row(b), G.LsamRows(z.data_ptr(), 0, 0), pw.data_ptr(), nw.data_ptr(), 0, 0)
    nbytes = G.lib().lsam_residual_norm_grad_workspace_bytes(G.FP32, 1, rows, n)
    ws, at = scratch(nbytes)
    err = C.create_string_buffer(256)
    torch.cuda.synchronize()
    rc = G.lib().lsam_selftest_residual_wait(r, row(x), fwd.rstd_post.data_ptr(), fwd.rstd_pre.data_ptr(), row(dy), row(du), row(got[0]), row(got[1]), G.LsamRows(got[2].data_ptr(), 0, 0),
                                             got[3].data_ptr(), got[4].data_ptr(), at, nbytes, torch.cuda.current_stream().cuda_stream, err, 256)
    assert rc == G.LSAM_OK, err.value
    torch.cuda.synchronize()
    ranks = 2 if n <= 8192 else 4 if n <= 16384 else 8
    share = -(-rows // (SMS // ranks))
    per = (-(-n // ranks) + 7) // 8 * 8
    place = torch.arange(rows, device="cuda") % share  # of a row in its block's share
    for a, w in zip(got[:2], want[:2]):
        nan = torch.isnan(a)
        assert (nan | (a == w)).all()  # nothing finite is wrong
        assert not nan[place < 2].any() and nan[place > 2].all() and nan[place == 2][:, :per].all() and not nan[place == 2][:, per:].any()
    # the first block writes the gradient of a gate per row
    assert torch.equal(got[2][place < 2], want[2][place < 2]) and torch.isnan(got[2][place >= 2]).all()
    # that of the norm's weight in front needs no sums over a row
    assert torch.isnan(got[3]).all() and torch.equal(got[4], want[4])
    again = G.lsam_residual_norm_grad(fwd, dy, du, act="sigmoid", **how)
    assert all(torch.equal(a, w) for a, w in zip(again, want))


# one CTA a tile, pairs, symmetric tiles with and without transposed ones, tall matrices, a Gram matrix that is shared out, several tiles a CTA
@pytest.mark.parametrize("K, rows, cols, steps", [(2, 40, 70, 1), (1, 128, 130, 2), (2, 300, 520, 2), (1, 777, 300, 1), (1, 128, 4096, 2), (3, 1100, 1100, 1), (40, 200, 210, 1)])
def test_operands_that_never_arrive(K, rows, cols, steps):
    g = torch.randn((K, rows, cols), generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda")
    want, got = G.lsam_orthogonalize(g), torch.full_like(g, 5.0)
    nbytes = G.lib().lsam_orthogonalize_workspace_bytes(G.FP32, K, rows, cols)
    ws, at = scratch(nbytes)
    err = C.create_string_buffer(256)
    torch.cuda.synchronize()
    size = rows * cols
    rc = G.lib().lsam_selftest_orthogonalize_wait(g.data_ptr(), G.FP32, K, rows, cols, size, cols, 1, steps, 3.4445, -4.775, 2.0315, 1.0, 1e-7, got.data_ptr(), size, cols, 1, at, nbytes,
                                                  torch.cuda.current_stream().cuda_stream, err, 256)
    assert rc == G.LSAM_OK, err.value
    torch.cuda.synchronize()
    assert torch.isnan(got).all()
    assert torch.equal(G.lsam_orthogonalize(g), want)
