"""What keeps the digits of a head's logits, each held by a bound that the call would miss without it: the three small products of an fp32 operand's planes, and
the chunks in which the tensor cores' sums are added.

u = 2^-24.  Model: a step of 16 inner indices cuts off at most two units in the last place of the accumulator (2 u each, of the sum so far).  With terms of one
sign the sum grows evenly, so n steps into one accumulator lose at most 2 * 2 u (n + 1) / 2 of its end; an accumulator takes 48 steps (768 inner indices) at
most.  Each chunk that is added rounds once.
"""
import pytest
import torch

from paper_2509_03110_b200 import binding as G
from test_gpu_head_ops import DT, U, close, grad_reference, make_labels, make_logits, reference

pytestmark = pytest.mark.gpu
STEPS = 48


def check(h, w, y, rel):
    """The scores against 64 bits, where a logit may be off by rel u of the sum of its terms' magnitudes."""
    l = h.double() @ w.double().transpose(-1, -2)
    mag = (h.double().abs() @ w.double().abs().transpose(-1, -2)).amax(-1)
    want = reference(l, y, 0)
    l_err = rel * U * mag
    r = G.lsam_head_logprob(h, w, y)
    close(r.lse, want["lse"], want["lse_err"] + l_err)
    return r.lse.double() - want["lse"], l_err, want["lse_err"]


def power(inner):
    """The power of two that brings a sum of `inner` ones to 32 .. 64, beside which the roundings of the scores themselves are small."""
    return 2.0 ** (5 - (inner.bit_length() - 1))


@pytest.mark.parametrize("rows", [9, 40, 200])
@pytest.mark.parametrize("inner, classes", [(100, 300), (128, 1000), (257, 77), (512, 300)])
def test_every_product_of_the_planes_counts(rows, inner, classes):
    # x = 1 + (2^-8 - 2^-16) + (2^-17 - j 2^-23): planes of 1, 2^-8 and 2^-17, all positive.  Without the product of the first and the third plane a sum is
    # 128 u short, without that of the second planes 256 u.  Left out on purpose: the second with the third, u together.
    g = torch.Generator(device="cuda").manual_seed(inner)
    draw = lambda *s: 1 + 2.0 ** -8 - 2.0 ** -17 - torch.randint(1, 9, s, generator=g, device="cuda").double() * 2.0 ** -23  # noqa: E731
    h, w = draw(2, rows, inner).float(), (draw(2, classes, inner) * power(inner)).float()
    p1 = (h - h.bfloat16().float()).bfloat16().float()
    assert (h.bfloat16() == 1).all() and (p1 == 2.0 ** -8 - 2.0 ** -16).all()
    steps, blocks = -(-inner // 16), -(-inner // 64)
    # (1,1) of the steps at full size; those of the second planes' products stand at 2^-8 of it and less: 2 u; the left-out products 2 u
    rel = 2 * (min(steps, STEPS) + 1) + 2 + 2 + -(-6 * blocks // 12)
    _, l_err, s_err = check(h, w, make_labels(2, rows, classes, 1), rel)
    assert (l_err + s_err < 128 * U * 32).all()  # what a missing product would cost at the least


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows", [16, 300])
def test_long_sums_of_one_sign_are_added_in_chunks(rows, dtype):
    # one accumulator for all 2048 steps would lose half a unit a step on average: 340 u at the least
    inner, classes = 32768, 70
    g = torch.Generator(device="cuda").manual_seed(rows)
    draw = lambda *s: 0.5 + torch.rand(s, generator=g, device="cuda")  # noqa: E731
    h, w = draw(1, rows, inner).to(DT[dtype]), (draw(1, classes, inner) * power(inner)).to(DT[dtype])
    rel = 2 * (STEPS + 1) + -(-inner // 768) + (6 if dtype == "fp32" else 0)
    diff, l_err, s_err = check(h, w, make_labels(1, rows, classes, 1), rel)
    assert (l_err + s_err < 340 * U * 16).all()
    assert (diff.mean().abs() <= (l_err + s_err).mean())


@pytest.mark.parametrize("layout", ["row", "feature", "strided"])
@pytest.mark.parametrize("size", [(1, 5, 1), (2, 9, 33), (2, 40, 1000), (1, 7, 2049), (1, 5, 20011)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_gradient_of_the_entropy_alone_without_labels(size, layout, dtype):
    K, rows, C = size
    l = make_logits(K, rows, C, dtype, layout, seed=C, pad=C % 3)
    if C > 1:
        l[0, 1, ::2] = float("-inf")
    l[0, 3] = float("-inf")
    r = G.lsam_logprob(l)
    b = torch.randn((K, rows), generator=torch.Generator(device="cuda").manual_seed(C), device="cuda")
    want, tol = grad_reference(l, None, r.lse, r.entropy, None, b)
    close(G.lsam_logprob_grad(l, None, r.lse, None, entropy=r.entropy, dentropy=b), want, tol)
    if C > 33:
        assert want.abs().max() > 0
