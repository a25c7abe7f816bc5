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
