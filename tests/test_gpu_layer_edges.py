"""Calls of the operators for layers and updates at the edge of what they take."""
import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, cols", [(1, 1), (9, 40), (32, 300), (150, 90), (300, 304)])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_what_is_not_finite_makes_its_whole_matrix_nan(rows, cols, steps, dtype):
    g = torch.randn((5, rows, cols), generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda").to(dtype)
    want = G.lsam_orthogonalize(g, steps=steps)
    for k, v in ((1, "inf"), (2, "-inf"), (4, "nan")):
        g[k, rows // 2, cols // 3] = float(v)
    got = G.lsam_orthogonalize(g, steps=steps)
    assert all(torch.isnan(got[k]).all() for k in (1, 2, 4)) and torch.equal(got[[0, 3]], want[[0, 3]])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gate", ["row", "column", "full", "none"])
def test_rows_of_no_columns(gate, dtype):
    K, rows = 3, 70
    x = torch.empty((K, rows, 0), device="cuda", dtype=dtype)
    w = torch.empty(0, device="cuda")
    z = {"row": torch.randn((K, rows, 1), device="cuda"), "column": w, "full": x.clone(), "none": None}[gate]
    junk = [torch.full((K, rows), 7.0, device="cuda") for _ in range(8)]  # what the results' memory holds before
    del junk
    r = G.lsam_residual_norm(x, branch=x.clone(), gate=z, post_weight=w, pre_weight=w)
    # the mean of no squares is 0 / 0, as torch has it
    assert r.out.shape == r.normed.shape == x.shape and torch.isnan(r.rstd_post).all() and torch.isnan(r.rstd_pre).all() and r.rstd_post.shape == (K, rows)
    junk = [torch.full((K, rows, 1), 7.0, device="cuda") for _ in range(8)]
    del junk
    d = G.lsam_residual_norm_grad(r, x, x, branch=x, gate=z, post_weight=w, pre_weight=w)
    assert d.dx.shape == d.dbranch.shape == x.shape and d.dpost_weight.shape == d.dpre_weight.shape == (0,)
    if gate == "row":  # a sum over no columns
        assert d.dgate.shape == z.shape and (d.dgate == 0).all()
        one = G.lsam_residual_norm_grad(r, x, None, branch=x, gate=z[:, :1].contiguous().expand(K, rows, 1).contiguous(), post_weight=w, act="sigmoid")
        assert (one.dgate == 0).all()
