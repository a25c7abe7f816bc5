"""Log-sum-exp in two words, and the gradient from it: against the 64-bit softmax of the logits themselves, however large the logits are.

u = 2^-24.  lse + lse_low: the sum of exponentials and its logarithm, as in the scores (s_err), and the roundings of log2 s, of the division and of ls: 4 u (1 + ls).
A probability: x = l - lse rounds once (u |x|), is scaled and exponentiated (4 u + 3 u |x| in all, as in the scores); e^-low is off by 2 u + u |low| and multiplied (2 u);
the two words' own error enters whole.
"""
import pytest
import torch

from paper_2509_03110_b200 import binding as G
from test_gpu_head_ops import DT, NAN, NINF, U, check_scores, close, grad_reference, make_labels, make_logits, reference

pytestmark = pytest.mark.gpu


def two_words(l):
    """64-bit log softmax and log-sum-exp (relative to the row's maximum), and the bound of the two words' error."""
    d = l.double()
    d = torch.where(d <= -1e30, torch.full_like(d, NINF), d)
    m = d.amax(-1, keepdim=True)
    m = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
    ls = (d - m).exp().sum(-1, keepdim=True).log()
    w = reference(l, None, 0)
    s_err = (l.shape[-1] / 8 + 68) * U + 3 * U * w["pu"]
    return d, m, ls, s_err + 4 * U * (1 + torch.nan_to_num(ls.squeeze(-1), 0, 0, 0).abs()), w


def check_gradient(l, y, a, b, r, got):
    d, m, ls, two_err, w = two_words(l)
    lp = (d - m) - ls
    p = lp.exp()
    live = p > 0
    H = w["entropy"].unsqueeze(-1)
    x = torch.where(live, (d - r.lse.double().unsqueeze(-1)).abs(), torch.zeros_like(d))  # what the kernel exponentiates
    low = r.lse_low.double().abs().unsqueeze(-1)
    rel = 4 * U + 3 * U * x + 4 * U + U * low + two_err.unsqueeze(-1) + 2 * U
    g, err = torch.zeros_like(d), torch.zeros_like(d)
    if a is not None:
        hot = (torch.arange(l.shape[-1], device="cuda") == y.unsqueeze(-1)).double()
        aa = a.double().unsqueeze(-1)
        g = g + aa * (hot - p)
        err = err + aa.abs() * (p * rel + 2 * U * hot)
    if b is not None:
        bb = b.double().unsqueeze(-1)
        xe = torch.where(live, lp + H, torch.zeros_like(lp))
        g = g - bb * p * xe
        # the terms b H, b low and b x are rounded and added; H and the two words carry their own errors
        err = err + bb.abs() * p * (xe.abs() * rel + 4 * U * (x + low + H.abs()) + two_err.unsqueeze(-1) + w["ent_err"].unsqueeze(-1))
    if a is not None and b is not None:
        err = err + 4 * U * p * a.double().abs().unsqueeze(-1)
    none = torch.isneginf(r.lse) if y is None else torch.isneginf(r.lse) | (y < 0)
    g, err = (torch.where(none.unsqueeze(-1), torch.zeros_like(t), t) for t in (g, err))
    fi = torch.finfo(l.dtype)
    close(got, g, err + 4 * U * g.abs() + fi.eps / 2 * g.abs() + fi.smallest_normal * fi.eps / 2 + 2.0 ** -126)


SIZES = [(2, 9, 1), (1, 9, 33), (2, 12, 1000), (1, 9, 2049), (1, 9, 20011), (1, 160, 9000)]
OFFSETS = [0.0, 1e3, -1e4, 1e6, 1e9, -1e9, 1e20, -1e29]


@pytest.mark.parametrize("layout", ["row", "feature", "strided"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_two_words_and_their_gradient_at_any_offset(size, layout):
    K, rows, C = size
    l = make_logits(K, rows, C, "fp32", layout, seed=C, pad=C % 3)
    for i, o in enumerate(OFFSETS):
        l[:, i] += o  # at 1e9 and beyond every class of the row is the same number
    if C > 4:
        l[0, 1, 3], l[0, 4, ::2] = NINF, NINF
    l[:, 8] = NINF
    y = make_labels(K, rows, C, C)
    y[K - 1, 2] = -1
    r = check_scores(l, y, 0)
    d, m, ls, two_err, _ = two_words(l)
    left = y < 0
    both = (r.lse.double() - m.squeeze(-1)) + r.lse_low.double()  # exact in 64 bits but where the offset is beyond them
    want = torch.where(left, torch.zeros_like(both), ls.squeeze(-1))
    both = torch.where(left, r.lse.double() + r.lse_low.double(), both)
    close(both, want, two_err + 2.0 ** -52 * 64)
    assert not r.lse_low[:, 8].any() and not r.lse_low[left].any()
    g = torch.Generator(device="cuda").manual_seed(C)
    a, b = (torch.randn((K, rows), generator=g, device="cuda") for _ in range(2))
    for aa, bb in ((a, None), (None, b), (a, b)):
        check_gradient(l, y, aa, bb, r, G.lsam_logprob_grad(l, y, r, aa, dentropy=bb))
    # the gradient of a cross-entropy sums to zero over a row
    total = G.lsam_logprob_grad(l, y, r, torch.ones_like(a)).double().sum(-1).abs()
    x = torch.where(torch.isfinite(d), (d - r.lse.double().unsqueeze(-1)).abs(), torch.zeros_like(d))
    p = torch.nan_to_num(((d - m) - ls).exp(), 0, 0, 0)
    bound = two_err + (p * (14 * U + 3 * U * x + 2 * U * r.lse_low.double().abs().unsqueeze(-1))).sum(-1) + 4 * U
    assert (total <= torch.where(left | torch.isneginf(r.lse), torch.zeros_like(bound), bound)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["row", "feature"])
def test_gradient_of_large_16_bit_logits(dtype, layout):
    l = make_logits(2, 40, 1500, dtype, layout, seed=5)
    l += torch.tensor([0.0, 40.0, -300.0, 3e3, 6e4], device="cuda").to(DT[dtype]).repeat(8).unsqueeze(-1)
    y = make_labels(2, 40, 1500, 3)
    r = check_scores(l, y, 0)
    a, b = torch.rand_like(r.lse), torch.rand_like(r.lse)
    check_gradient(l, y, a, b, r, G.lsam_logprob_grad(l, y, r, a, dentropy=b))
    check_gradient(l, y, a, None, r, G.lsam_logprob_grad(l, y, r.lse, a, lse_low=r.lse_low))


def test_one_word_is_the_documented_form():
    # lse alone, as before: p = e^(l - lse) with the rounded lse; and in two words with a low word of zero, the same bits
    l = make_logits(1, 30, 777, "fp32", "row", seed=2)
    l[0, :10] += 100.0
    y = make_labels(1, 30, 777, 2)
    r = G.lsam_logprob(l, y)
    a, b = torch.rand_like(r.lse), torch.rand_like(r.lse)
    one = G.lsam_logprob_grad(l, y, r.lse, a, entropy=r.entropy, dentropy=b)
    want, tol = grad_reference(l, y, r.lse, r.entropy, a, b)
    close(one, want, tol)
    assert torch.equal(one, G.lsam_logprob_grad(l, y, r.lse, a, entropy=r.entropy, dentropy=b, lse_low=torch.zeros_like(a)))
    # the documented size of what one word loses: a factor of 1 +- |lse| u on every p
    two = G.lsam_logprob_grad(l, y, r, a)
    one = G.lsam_logprob_grad(l, y, r.lse, a)
    p = torch.log_softmax(l.double(), -1).exp()
    x = (l.double() - r.lse.double().unsqueeze(-1)).abs()
    loss = a.double().unsqueeze(-1) * (p * (1.01 * U * r.lse.double().abs().unsqueeze(-1) + 30 * U + 8 * U * x + (777 / 8 + 80) * U) + 4 * U)
    assert ((one.double() - two.double()).abs() <= loss).all()


def test_an_emptied_row_has_a_gradient_that_sums_to_zero():
    # every class behind an additive mask of -1e9: not a mask by the rule, a uniform row of 1000 classes
    for C in (40, 1000, 5003):
        l = torch.full((1, 2, C), -1e9, device="cuda")
        y = torch.zeros((1, 2), device="cuda", dtype=torch.int32)
        r = G.lsam_logprob(l, y)
        d = G.lsam_logprob_grad(l, y, r, torch.ones_like(r.lse), dentropy=torch.ones_like(r.lse))
        want = torch.full((1, 2, C), -1.0 / C, device="cuda", dtype=torch.float64)
        want[..., 0] += 1
        # p is off by the two words' error (C / 8 + 68 + 4 (1 + log C)) u, the entropy's term (log p + H = 0) by p times a few u (log C)^2
        tol = ((C / 8 + 80 + 40) * U + 60 * U * 3) / C + 4 * U * want.abs()
        close(d, want, tol)


def test_a_row_of_nan_and_refusals():
    l = make_logits(1, 3, 50, "fp32", "row", seed=1)
    l[0, 1, 7] = NAN
    y = torch.tensor([[1, 2, -1]], device="cuda", dtype=torch.int32)
    r = G.lsam_logprob(l, y)
    d = G.lsam_logprob_grad(l, y, r, torch.ones_like(r.lse))
    assert torch.isnan(r.lse_low[0, 1]) and torch.isnan(d[0, 1]).all() and torch.isfinite(d[0, 0]).all() and not d[0, 2].any()
    assert G.lsam_head_logprob(l, l).lse_low is None and len(r) == 5
    for bad in (r.lse_low.double(), r.lse_low[:, :2], r.lse_low.cpu()):
        with pytest.raises(G.LsamError) as e:
            G.lsam_logprob_grad(l, y, r.lse, torch.ones_like(r.lse), lse_low=bad)
        assert e.value.code == G.LSAM_ERR_INVALID
