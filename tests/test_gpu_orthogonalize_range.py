"""Orthogonalisation of matrices whose norm lies in few rows, elements or directions, with more steps and with other polynomials, in every type.

Bound.  Errors are carried on by the later steps, more or less by the matrix and the polynomial, so what a result may be off by is what the 64-bit steps and a plain chain say of the same matrix:
- The planes hold an element to 2^-24 and leave out 2^-24 of every term, a chain of fp32 products rounds every element and sum to 2^-24.  The signs of both are anything: 8 times the chain's error.
- The accumulators cut off towards zero: 12 steps of 16 indices a chunk, those of the small products at their own size, so at most 4 + 1 times 2^-23 of a sum of positive terms, in every
  product the same way.  That is what the 64-bit steps do with every product times 1 - 2^-20.
- Where both happen to be exact (a single element), 2^-24 for each product of each step.
What is stored in 16 bits may be off by half a step of its type beyond that, element by element."""
import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)
POLYNOMIALS = [(ABC, 5), (ABC, 10), ((4.0848, -6.8946, 2.9270), 5), ((3.0, -4.0, 1.0), 8), ((4.0, -6.0, 2.5), 2), ((2.5, -2.5, 0.0), 16), ((1.875, -1.25, 0.375), 12)]


def steps(g, abc, n, scale, dtype, cut=0.0):
    """The steps as a chain of plain products in `dtype`, each of them times 1 - cut."""
    f = 1.0 - cut
    a, b, c = (float(torch.tensor(v, dtype=torch.float32)) for v in abc)
    x = g.double()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = (x / (x.flatten(1).norm(dim=1).view(-1, 1, 1) + 1e-7)).to(dtype)
    for _ in range(n):
        m = f * (x @ x.transpose(1, 2))
        x = a * x + f * ((b * m + c * f * (m @ m)) @ x)
    x = scale * x
    return (x.transpose(1, 2) if tall else x).double()


def half_step(v, t):
    """Half of the distance of neighbouring numbers of a type at v."""
    e = torch.finfo(t)
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=e.tiny)))) * (e.eps / 2)


def beyond(got, ref):
    """How far the result is from the exact one beyond what its own rounding explains."""
    t = got.dtype
    return ((got.double() - ref).abs() - torch.maximum(half_step(got.double(), t), half_step(ref, t))).clamp(min=0)


def matrix(kind, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = torch.zeros((2, rows, cols), device="cuda")
    if kind == "normal":
        x = rand(2, rows, cols)
    elif kind == "rows":  # rare tokens, idle units
        x[:, 3:rows:rows // 8] = rand(*x[:, 3:rows:rows // 8].shape)
    elif kind == "columns":
        x[..., 5:cols:cols // 3] = rand(*x[..., 5:cols:cols // 3].shape)
    elif kind == "element":
        x[:, rows - 2, 17] = torch.tensor([1.7, -0.3], device="cuda")
    elif kind == "diagonal":
        i = torch.arange(8, device="cuda") * (min(rows, cols) // 8)
        x[:, i, i] = rand(2, 8)
    elif kind == "constant":
        x[0], x[1] = 1.1, -0.013
    else:  # "one": a direction that holds most of the norm, over a floor
        x = rand(2, rows, 1) @ rand(2, 1, cols) + 0.1 * rand(2, rows, cols)
    return (x * 1e-2).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["normal", "rows", "columns", "element", "diagonal", "constant", "one"])
@pytest.mark.parametrize("rows, cols", [(512, 512), (600, 1100), (2050, 520), (100, 130)])
def test_whatever_the_norm_lies_in(rows, cols, kind, dtype):
    g = matrix(kind, rows, cols, dtype)
    for abc, n in POLYNOMIALS:
        got = G.lsam_orthogonalize(g, steps=n, coefficients=abc, scale=1.5)
        ref = steps(g, abc, n, 1.5, torch.float64)
        size = lambda v: v.flatten(1).norm(dim=1)  # noqa: E731
        bound = 8 * size(steps(g, abc, n, 1.5, torch.float32) - ref) + size(steps(g, abc, n, 1.5, torch.float64, 2.0 ** -20) - ref) + 3 * n * 2.0 ** -24 * size(ref)
        err = size(beyond(got, ref))
        assert got.dtype == dtype and (err <= bound).all(), (abc, n, (err / size(ref)).tolist(), (err / bound).tolist())
        # The products are the same whatever the type.  (The norm's sum in double may take its terms in another order: a relative 2^-50 of X, which moves one element in 2^26 to the
        # neighbouring fp32 number.  Were all of them moved, 2^-24 of 2^-11, the fp16 numbers' distance, could come out on the other side of a border, one in 2^13.)
        wide = G.lsam_orthogonalize(g.float(), steps=n, coefficients=abc, scale=1.5).to(dtype)
        assert (got != wide).double().mean() <= 2.0 ** -13, (abc, n)
