"""The operators around a classifier's head against their definitions in 64 bits, at the sizes, layouts and masks where they can go wrong.

Where the tolerances come from (u = 2^-24, half a step of fp32).  e^x is 2^(x log2 e) on the special-function unit: the result is off by at
most 2^-22, the argument by half a step of |x| and of |x log2 e|, together a relative error of at most 4 u + 3 u |x| =: d(x).
A sum of n positive terms held by at least 8 threads in sequence and joined by a tree or in order: at most (n / 8 + 64) u.
"""
import numpy as np
import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
NINF, NAN, INF = float("-inf"), float("nan"), float("inf")


def make_logits(K, rows, C, dtype, layout, seed, scale=2.5, pad=0):
    """A [K, rows, C] tensor stored as rows, with the sample index contiguous, or with no unit stride at all."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = (torch.randn((K, rows, C), generator=g, device="cuda") * scale).to(DT[dtype])
    if layout == "row":
        t = torch.empty((K, rows, C + pad), device="cuda", dtype=DT[dtype])[:, :, pad:]
    elif layout == "feature":
        t = torch.empty((K, C, rows + pad), device="cuda", dtype=DT[dtype])[:, :, :rows].transpose(1, 2)
    else:
        t = torch.empty((K, rows, C, 3), device="cuda", dtype=DT[dtype])[..., 1]
    t.copy_(v)
    return t


def reference(l, labels, top_k):
    """Scores in 64 bits of the stored values, and the bounds of their errors."""
    C = l.shape[-1]
    d = l.double()
    d = torch.where(d <= -1e30, torch.full_like(d, NINF), d)  # masks
    m = torch.where(torch.isnan(d), torch.full_like(d, NINF), d).amax(-1, keepdim=True)
    base = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
    z = (d - base).exp().sum(-1, keepdim=True).log()  # a +inf logit makes it NaN
    lse = (base + z).squeeze(-1)
    lp = (d - base) - z  # relative to the maximum: exact where lse is so large that it swallows log z
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, torch.zeros_like(p))).sum(-1)
    empty = torch.isneginf(lse)
    ent = torch.where(empty, torch.zeros_like(ent), ent)
    pu = torch.where(p > 0, p * (d - m).abs(), torch.zeros_like(p)).sum(-1)  # E|l - m|
    pu2 = torch.where(p > 0, p * (d - m) ** 2, torch.zeros_like(p)).sum(-1)
    s_err = (C / 8 + 68) * U + 3 * U * pu                                    # relative error of sum e^(l - m)
    fin = lambda t: torch.where(torch.isfinite(t), t, torch.zeros_like(t))   # noqa: E731
    lse_err = s_err + 4 * U * (1 + fin(lse).abs())
    ent_err = s_err * (2 + 2 * pu) + 4 * U * (2 + pu + pu2) + 4 * U * fin(ent).abs()
    out = dict(lse=lse, entropy=ent, lse_err=lse_err, ent_err=ent_err, pu=pu)
    if labels is not None:
        left = labels < 0
        lab = labels.clamp(min=0, max=C - 1).long().unsqueeze(-1)
        at = d.gather(-1, lab).squeeze(-1)
        logp = torch.where(torch.isneginf(at), at, lp.gather(-1, lab).squeeze(-1))
        logp = torch.where(labels >= C, torch.full_like(logp, NAN), logp)
        out["logp"] = torch.where(left, torch.zeros_like(logp), logp)
        for k in ("lse", "entropy"):
            out[k] = torch.where(left, torch.zeros_like(out[k]), out[k])
    if top_k:
        rank = torch.where(torch.isnan(d), torch.full_like(d, NINF), d)
        if labels is not None:
            rank = torch.where((labels < 0).unsqueeze(-1), torch.full_like(rank, NINF), rank)
        v, i = torch.sort(rank, dim=-1, descending=True, stable=True)
        kk = min(top_k, C)
        tv = torch.full((*l.shape[:-1], top_k), NINF, device=l.device, dtype=torch.float64)
        ti = torch.full((*l.shape[:-1], top_k), -1, device=l.device, dtype=torch.int32)
        none = torch.isneginf(v[..., :kk])
        tv[..., :kk] = torch.where(none, v[..., :kk], lp.gather(-1, i[..., :kk]))
        ti[..., :kk] = torch.where(none, torch.full_like(i[..., :kk], -1), i[..., :kk]).int()
        out["top_logp"], out["top_idx"] = tv, ti
    return out


def close(got, want, tol):
    """Equal where not finite, within tol elsewhere."""
    got, want = got.double().cpu().numpy(), want.cpu().numpy()
    tol = np.broadcast_to(tol.cpu().numpy() if isinstance(tol, torch.Tensor) else tol, want.shape)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine])
    bad = ~(np.abs(got[fine] - want[fine]) <= tol[fine])  # a NaN is never within
    assert not bad.any(), (got[fine][bad][:5], want[fine][bad][:5], tol[fine][bad][:5])


def check_scores(l, labels, top_k, r=None):
    r = r or G.lsam_logprob(l, labels, top_k=top_k)
    w = reference(l, labels, top_k)
    close(r.lse, w["lse"], w["lse_err"])
    close(r.entropy, w["entropy"], w["ent_err"])
    if labels is not None:
        close(r.logp, w["logp"], w["lse_err"] + 2 * U * torch.nan_to_num(w["logp"], 0, 0, 0).abs())
    if top_k:
        assert torch.equal(r.top_idx, w["top_idx"])
        close(r.top_logp, w["top_logp"], (w["lse_err"] + 4 * U).unsqueeze(-1) + 2 * U * torch.nan_to_num(w["top_logp"], 0, 0, 0).abs())
    return r


def make_labels(K, rows, C, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    return torch.randint(0, C, (K, rows), generator=g, device="cuda", dtype=torch.int32)


SIZES = [(1, 1, 1), (1, 1, 2), (2, 3, 7), (1, 9, 31), (1, 5, 33), (3, 33, 100), (2, 40, 1000), (1, 3, 1025), (1, 7, 2049), (2, 5, 4097), (1, 2, 8200), (1, 3, 50021), (1, 2, 131073)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["row", "feature", "strided"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_scores(size, layout, dtype):
    K, rows, C = size
    l = make_logits(K, rows, C, dtype, layout, seed=C, pad=C % 3)
    y = make_labels(K, rows, C, C)
    y[0, 0] = -1
    if rows > 2:
        y[0, 2] = C
    check_scores(l, y, [0, 1, 5, 8, 20, 32][(C + rows) % 6])
    check_scores(l, None, 3)


@pytest.mark.parametrize("layout, rows, C", [("row", 5000, 10), ("row", 4097, 64), ("feature", 33000, 17), ("feature", 40000, 100), ("feature", 32768, 256), ("strided", 4100, 33)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_scores_of_many_short_rows(layout, rows, C, dtype):
    l = make_logits(1, rows, C, dtype, layout, seed=C, pad=C % 3)
    l[0, 1] = NINF
    l[0, 2, ::2] = NINF
    l[0, 3] = 0.0
    l[0, 4, C // 2] = NAN
    l[0, 5] = torch.finfo(DT[dtype]).min if dtype != "fp16" else NINF
    y = make_labels(1, rows, C, C)
    y[0, 0], y[0, rows - 1], y[0, 6] = -1, -7, C
    for k in (0, 1, 5, 32):
        check_scores(l, y, k)


@pytest.mark.parametrize("layout", ["row", "feature"])
@pytest.mark.parametrize("C", [10, 257, 1000, 4100, 40001])
def test_scores_of_masked_rows(C, layout):
    rows = 16
    l = make_logits(1, rows, C, "fp32", layout, seed=3)
    l[0, 0] = NINF                       # nothing left
    l[0, 1] = NINF; l[0, 1, C // 2] = 1.5  # one class left
    l[0, 2, ::2] = NINF
    l[0, 3] = torch.finfo(torch.float32).min
    l[0, 4, 1:] = torch.finfo(torch.float32).min
    l[0, 5, C - 1] = NAN
    l[0, 6, 0] = INF
    l[0, 7] = NAN
    l[0, 8] = INF
    l[0, 9] = 0.0                        # every class equal
    l[0, 10] = -0.0; l[0, 10, 1] = 0.0
    l[0, 11, :] = NINF; l[0, 11, 3] = NAN
    l[0, 12, 1:] = -1e9                  # usual masks, and whole rows of large numbers
    l[0, 13] = -1e10
    l[0, 14] = 2e38; l[0, 14, 0] = 1e38  # the documented end of the range
    l[0, 15] = NINF; l[0, 15, C - 2:] = 0.5  # a few classes at the end
    y = torch.full((1, rows), 1, device="cuda", dtype=torch.int32)
    for k in (1, 8, 32):
        check_scores(l, y, k)
    y[0, 7:9] = -5  # garbage in rows that are left out
    check_scores(l, y, 5)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [40, 1000, 6001, 70001])
def test_alternatives_of_tied_and_sorted_rows(C, dtype):
    # few distinct values, ascending and descending rows, one value repeated in the tail: the lower class wins every tie
    i = torch.arange(C, device="cuda")
    rows = [(i % 3).float(), (i % 2).float() * -1, i.float() / 64, -i.float() / 64, torch.zeros(C, device="cuda"), (i >= C - 40).float(), (i // 97 % 5).float(), -(i - C // 2).abs().float() / 8]
    l = torch.stack(rows)[None].to(DT[dtype])
    for k in (1, 7, 32):
        check_scores(l.contiguous(), None, k)
        check_scores(l.transpose(1, 2).contiguous().transpose(1, 2), None, k)


@pytest.mark.parametrize("K, rows", [(2, 17), (1, 3), (2, 32), (1, 148)])  # rows split over eight blocks and over four
@pytest.mark.parametrize("dtype, C", [("fp32", 20011), ("bf16", 33001)])
def test_ties_and_masks_in_split_rows(K, rows, dtype, C):
    g = torch.Generator(device="cuda").manual_seed(rows)
    l = torch.randint(-3, 3, (K, rows, C), generator=g, device="cuda").to(DT[dtype])
    l[0, 0] = NINF
    l[0, 1] = NINF; l[0, 1, C - 3:] = 2.0
    l[0, 2] = -1.0
    l[K - 1, rows - 1, ::2] = torch.finfo(DT[dtype]).min
    l[K - 1, 0, C // 2] = NAN if K > 1 else 9.0
    y = make_labels(K, rows, C, 1)
    y[0, 1], y[K - 1, 2] = C - 1, -1
    for k in (0, 1, 9, 32):
        check_scores(l, y, k)


def test_scores_beyond_32_bit_offsets():
    stride = (1 << 31) + 8
    C = 1000
    flat = torch.empty(stride + C, device="cuda", dtype=torch.bfloat16)
    l = flat.as_strided((1, 2, C), (0, stride, 1))
    l.copy_(torch.randn((1, 2, C), device="cuda") * 3)
    y = torch.tensor([[5, 999]], device="cuda", dtype=torch.int32)
    r = check_scores(l, y, 8)
    out = G.lsam_logprob_grad(l, y, r.lse, torch.ones_like(r.lse), out=l)  # in place
    assert out.data_ptr() == l.data_ptr() and float(l[0, 1].float().abs().sum()) > 0


def test_expanded_logits_and_unaligned_addresses():
    base = torch.randn(5003, device="cuda").bfloat16()
    for off in range(1, 9):  # every misalignment of a 16-byte vector
        l = base[off:off + 4990][None, None].expand(1, 3, 4990)
        check_scores(l, make_labels(1, 3, 4990, off), 5)


def grad_reference(l, y, lse, ent, a, b):
    d = l.double()
    x = d - lse.double().unsqueeze(-1)
    p = x.exp()
    g = torch.zeros_like(d)
    err = torch.zeros_like(d)
    rel = 4 * U + 3 * U * torch.where(p > 0, x.abs(), torch.zeros_like(x)) + U
    if a is not None:
        hot = (torch.arange(l.shape[-1], device="cuda") == y.unsqueeze(-1)).double()
        g = g + a.double().unsqueeze(-1) * (hot - p)
        err = err + a.double().abs().unsqueeze(-1) * (p * rel + 2 * U * hot)
    if b is not None:
        xe = torch.where(p > 0, x + ent.double().unsqueeze(-1), torch.zeros_like(x))
        g = g - b.double().unsqueeze(-1) * p * xe
        err = err + b.double().abs().unsqueeze(-1) * p * (xe.abs() * (rel + 2 * U) + 3 * U * (torch.where(p > 0, x.abs(), torch.zeros_like(x)) + ent.double().abs().unsqueeze(-1)))
    none = torch.isneginf(lse)  # nothing but masks
    none = none if y is None else none | (y < 0)
    g = torch.where(none.unsqueeze(-1), torch.zeros_like(g), g)
    err = torch.where(none.unsqueeze(-1), torch.zeros_like(err), err)  # exactly zero there, whatever the logits hold
    if y is not None:
        g = torch.where((y >= l.shape[-1]).unsqueeze(-1), torch.full_like(g, NAN), g)
    fi = torch.finfo(l.dtype)
    return g, err + 4 * U * g.abs().nan_to_num() + fi.eps / 2 * g.abs().nan_to_num() + fi.smallest_normal * fi.eps / 2 + 2.0 ** -126


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["row", "feature", "strided"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(size, layout, dtype):
    K, rows, C = size
    l = make_logits(K, rows, C, dtype, layout, seed=C + 1, pad=(C + 1) % 3)
    if rows > 3:
        l[0, 1] = NINF
        l[0, 3, ::3] = NINF
    if rows > 4:
        l[0, 4] = torch.finfo(DT[dtype]).min
    y = make_labels(K, rows, C, C)
    if rows > 2:
        y[0, 0] = -1
        l[0, 0, 0] = NAN
        y[0, 2] = C
    r = G.lsam_logprob(l, y)
    g = torch.Generator(device="cuda").manual_seed(C)
    a = torch.randn((K, rows), generator=g, device="cuda")
    b = torch.randn((K, rows), generator=g, device="cuda")
    for aa, bb in ((a, None), (None, b), (a, b)):
        got = G.lsam_logprob_grad(l, y, r.lse, aa, entropy=r.entropy if bb is not None else None, dentropy=bb)
        want, tol = grad_reference(l, y, r.lse, r.entropy, aa, bb)
        close(got, want, tol)
    got = G.lsam_logprob_grad(l, None, torch.where(y < 0, torch.zeros_like(r.lse), r.lse), None, entropy=r.entropy, dentropy=b)
    assert got.shape == l.shape


def test_gradient_into_other_strides_and_in_place():
    l = make_logits(2, 33, 130, "fp32", "row", seed=1)
    y = make_labels(2, 33, 130, 2)
    r = G.lsam_logprob(l, y)
    a = torch.rand_like(r.lse)
    want = G.lsam_logprob_grad(l, y, r.lse, a)
    feat = torch.zeros((2, 130, 48), device="cuda")
    view = feat[:, :, :33].transpose(1, 2)
    G.lsam_logprob_grad(l, y, r.lse, a, out=view)
    assert torch.equal(view, want) and not feat[:, :, 33:].any()
    lf = feat.clone()[:, :, :33].transpose(1, 2)
    lf.copy_(l)
    row = torch.full((2, 33, 140), 7.0, device="cuda")
    G.lsam_logprob_grad(lf, y, r.lse, a, out=row[:, :, :130])
    assert torch.equal(row[:, :, :130], want) and (row[:, :, 130:] == 7).all()
    G.lsam_logprob_grad(l, y, r.lse, a, out=l)
    assert torch.equal(l, want)


def test_gradient_of_empty_rows_and_expanded_logits():
    for C in (33, 2000):
        l = torch.full((1, 3, C), NINF, device="cuda")
        l[0, 2] = 0.5
        y = torch.tensor([[C, 1, C]], device="cuda", dtype=torch.int32)
        r = G.lsam_logprob(l, y)
        for t in (l, l.transpose(1, 2).contiguous().transpose(1, 2)):
            d = G.lsam_logprob_grad(t, y, r.lse, torch.ones_like(r.lse))
            assert not d[0, :2].any() and torch.isnan(d[0, 2]).all()  # nothing but masks comes before a label that is no class
        base = torch.randn((1, 1, C), generator=torch.Generator(device="cuda").manual_seed(C), device="cuda")
        e = base.expand(2, 5, C)
        y = make_labels(2, 5, C, C)
        r = check_scores(e, y, 3)
        want, tol = grad_reference(e, y, r.lse, r.entropy, torch.ones_like(r.lse), None)
        close(G.lsam_logprob_grad(e, y, r.lse, torch.ones_like(r.lse)), want, tol)


def test_gradient_against_differences():
    # of the 64-bit loss sum a logp + b entropy, along random directions: a central difference of step h is off by h^2 / 6 |L'''| <= 1e-9 here
    l = make_logits(1, 6, 50, "fp32", "row", seed=9, scale=1.0)
    y = make_labels(1, 6, 50, 9)
    r = G.lsam_logprob(l, y)
    a, b = torch.linspace(-1, 1, 6, device="cuda")[None], torch.linspace(2, -1, 6, device="cuda")[None]
    g = G.lsam_logprob_grad(l, y, r.lse, a, entropy=r.entropy, dentropy=b)

    def loss(d):
        lp = torch.log_softmax(d, -1)
        return (a.double() * lp.gather(-1, y.long().unsqueeze(-1)).squeeze(-1) - b.double() * (lp.exp() * lp).sum(-1)).sum()

    for s in range(4):
        v = torch.randn(l.shape, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").double()
        v /= v.norm()
        h = 1e-4
        diff = (loss(l.double() + h * v) - loss(l.double() - h * v)) / (2 * h)
        _, tol = grad_reference(l, y, r.lse, r.entropy, a, b)
        # lse and entropy themselves are rounded: relative change of p by half a step of lse, of the entropy term by its own error
        w = reference(l, y, 0)
        slack = (tol.norm() + (a.abs() + 4 * b.abs()).norm() * (w["lse_err"].max() + w["ent_err"].max()) + 1e-8).item()
        assert abs((g.double() * v).sum().item() - diff.item()) <= slack


def head_reference(h, w, bias, y):
    l = h.double() @ w.double().transpose(-1, -2)
    mag = h.double().abs() @ w.double().abs().transpose(-1, -2)
    if bias is not None:
        l = l + (bias.double().unsqueeze(-2) if bias.dim() == 2 else bias.double())
    l = torch.where(l <= -1e30, torch.full_like(l, NINF), l)
    # fp32 accumulation, in the tensor cores with truncated addends: at most one step of the running magnitude per term
    l_err = (2 * U * (h.shape[-1] + 8) * mag).amax(-1)
    out = reference(l, y, 0)
    out["lse_err"] = out["lse_err"] + l_err
    out["ent_err"] = out["ent_err"] + 2 * l_err * (1 + out["pu"]) * 2
    out["l_err"] = l_err
    return out


HEADS = [(1, 1, 8, 1), (1, 1, 64, 40), (2, 3, 40, 130), (1, 130, 72, 300), (3, 65, 100, 1000), (1, 257, 128, 1000), (2, 129, 264, 513), (1, 5, 1001, 77), (1, 300, 512, 5003), (2, 256, 96, 2048), (1, 2, 24, 20011),
         (2, 7, 1001, 3000), (1, 8, 6500, 300), (1, 1, 4100, 999), (3, 4, 257, 130), (2, 100, 1003, 777), (1, 150, 2050, 301)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("size", HEADS, ids=lambda s: "x".join(map(str, s)))
def test_head_scores(size, dtype):
    K, rows, D, C = size
    g = torch.Generator(device="cuda").manual_seed(C)
    h = torch.randn((K, rows, D), generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn((K, C, D), generator=g, device="cuda") * 2 / D ** 0.5).to(DT[dtype])
    bias = torch.randn((K, C), generator=g, device="cuda")
    y = make_labels(K, rows, C, C)
    y[0, 0] = C if rows > 1 else 0
    y[0, rows // 2] = -1 if rows > 1 else C - 1
    if C > 4:
        bias[:, 3] = NINF  # a masked class
    for ww, bb in ((w, None), (w, bias), (w[0], bias[0])):
        ws = torch.cuda.memory_allocated()
        r = G.lsam_head_logprob(h, ww, y, bias=bb)
        assert torch.cuda.memory_allocated() - ws < 1 << 20  # the workspace is given back
        t = head_reference(h, ww, bb, y)
        close(r.lse, t["lse"], t["lse_err"])
        close(r.entropy, t["entropy"], t["ent_err"])
        close(r.logp, t["logp"], t["lse_err"] + t["l_err"] + 4 * U * torch.nan_to_num(t["logp"], 0, 0, 0).abs())
    r = G.lsam_head_logprob(h, w)
    assert r.logp is None and torch.isfinite(r.lse).all()


def test_head_scores_of_strided_and_masked_operands():
    g = torch.Generator(device="cuda").manual_seed(0)
    for off, stride in ((0, 136), (8, 144), (1, 137), (3, 160)):  # tensor-core alignment and not
        h = torch.randn((2, 70, stride), generator=g, device="cuda").bfloat16()[:, :, off:off + 128]
        w = (torch.randn((2, 333, stride), generator=g, device="cuda") * 0.2).bfloat16()[:, :, off:off + 128]
        y = make_labels(2, 70, 333, off)
        bias = torch.full((2, 333), NINF, device="cuda")  # worker 0: nothing left; worker 1: two classes left
        bias[1, 5], bias[1, 300] = 0.5, 0.25
        r = G.lsam_head_logprob(h, w, y, bias=bias)
        t = head_reference(h, w, bias, y)
        close(r.lse, t["lse"], t["lse_err"])
        close(r.entropy, t["entropy"], t["ent_err"])
        close(r.logp, t["logp"], t["lse_err"] + t["l_err"])
        h[0, 1, 3] = NAN
        h[1, 2, 0] = INF
        r = G.lsam_head_logprob(h, w, y)
        assert torch.isnan(r.lse[0, 1]) and not torch.isfinite(r.lse[1, 2]) and torch.isfinite(r.lse[0, 2:]).all() and torch.isfinite(r.lse[1, 3:]).all()


def check_head(h, w, y, bias=None):
    r = G.lsam_head_logprob(h, w, y, bias=bias)
    t = head_reference(h, w, bias, y)
    close(r.lse, t["lse"], t["lse_err"])
    close(r.entropy, t["entropy"], t["ent_err"])
    close(r.logp, t["logp"], t["lse_err"] + t["l_err"] + 4 * U * torch.nan_to_num(t["logp"], 0, 0, 0).abs())


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 5, 70, 200])
def test_head_scores_of_permuted_and_expanded_operands(rows, dtype):
    K, C, D = 3, 300, 136
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    h, w = rand(K, rows, D).to(DT[dtype]), (rand(K, C, D) / 8).to(DT[dtype])
    y = make_labels(K, rows, C, rows)
    hp, wp = h.transpose(0, 1).contiguous().transpose(0, 1), w.transpose(0, 1).contiguous().transpose(0, 1)  # the workers' stride below the rows'
    check_head(hp, wp, y)
    check_head(h, wp, y, bias=rand(K, C))
    check_head(h[:1].expand(K, rows, D), w, y)               # one batch for all workers
    check_head(h[:, :1].expand(K, rows, D), w[0], y)         # one row, read again
    check_head(h, w[:, :1].expand(K, C, D), y)               # every class the same
    check_head(h, w[:1].expand(K, C, D), y, bias=rand(C))    # a shared head as an expanded tensor
    flat = (rand(C * 8 + D) / 8).to(DT[dtype])
    check_head(h, flat.as_strided((C, D), (8, 1)), y)        # classes whose rows overlap


def test_head_scores_of_more_rows_than_a_grid_of_tiles():
    g = torch.Generator(device="cuda").manual_seed(0)
    rows = 65535 * 32 + 40
    check_head(torch.randn((1, rows, 2), generator=g, device="cuda"), torch.randn((3, 2), generator=g, device="cuda"), make_labels(1, rows, 3, 0))


def test_head_scores_agree_with_scores_of_stored_logits():
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn((1, 200, 256), generator=g, device="cuda").half()
    w = (torch.randn((1, 1500, 256), generator=g, device="cuda") / 8).half()
    y = make_labels(1, 200, 1500, 1)
    l = (h.double() @ w.double().transpose(1, 2)).float()
    a, b = G.lsam_head_logprob(h, w, y), G.lsam_logprob(l, y)
    t = head_reference(h, w, None, y)
    for p, q in ((a.logp, b.logp), (a.lse, b.lse)):
        assert ((p - q).abs() <= 2 * t["lse_err"] + t["l_err"] + 8 * U * q.abs()).all()


# ------------------------------------------------------------------------------------------------ dropout
def philox(c, k):
    """Philox4x32-10 on uint64 arrays that hold 32-bit words, from its published definition."""
    c, k = [np.asarray(v, np.uint64) for v in c], list(k)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        s, m = np.uint64(32), np.uint64(0xFFFFFFFF)
        c = [(p1 >> s) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> s) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(K, rows, n, p, seed, tick, layer, k_offset):
    groups = -(-n // 8)
    g, r, k = np.meshgrid(np.arange(groups), np.arange(rows), np.arange(K), indexing="ij")
    w = philox([g, r, k + k_offset + (layer << 20), np.full(g.shape, tick & 0xFFFFFFFF)], [(seed & 0xFFFFFFFF) ^ 0x64726F70, (seed >> 32) ^ (tick >> 32)])
    bits = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1)  # [groups, rows, K, 8]
    bits = bits.transpose(2, 1, 0, 3).reshape(K, rows, groups * 8)[:, :, :n].astype(np.int64)
    return bits >= int(np.floor(p * 65536 + 0.5))


def test_philox_of_the_reference_mask_matches_the_published_vectors():
    import os

    n = 0
    for line in open(os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.txt")):
        words = [t for t in line.replace(":", " ").split() if len(t) == 8 and all(ch in "0123456789abcdefABCDEF" for ch in t)]
        if len(words) == 10:
            v = [int(t, 16) for t in words]
            assert [int(t) for t in philox(v[:4], v[4:6])] == v[6:]
            n += 1
    assert n >= 1


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("size, pad, off", [((1, 1, 1), 0, 0), ((1, 1, 8), 0, 0), ((2, 3, 7), 1, 1), ((3, 5, 9), 7, 0), ((1, 4, 1000), 8, 8), ((4, 33, 1021), 3, 2), ((2, 7, 4096), 0, 0), ((1, 300, 64), 0, 0), ((1, 2, 20001), 0, 0)],
                         ids=lambda v: str(v))
@pytest.mark.parametrize("with_skip", [False, True])
def test_dropout(size, pad, off, dtype, with_skip):
    K, rows, n = size
    g = torch.Generator(device="cuda").manual_seed(n)
    mk = lambda: torch.randn((K, rows, n + pad), generator=g, device="cuda").to(DT[dtype])[:, :, min(off, pad):min(off, pad) + n]  # noqa: E731
    x, skip = mk(), mk() if with_skip else None
    p, seed, tick, layer, k0 = 0.3, 0xFEDCBA9876543210, (5 << 32) + 77, 11, 5
    keep = torch.from_numpy(keep_mask(K, rows, n, p, seed, tick, layer, k0)).cuda()
    cut = int(np.floor(p * 65536 + 0.5))
    xs = x.double() * (65536 / (65536 - cut))
    want = torch.where(keep, xs, torch.zeros_like(xs)) + (skip.double() if with_skip else 0)
    mag = torch.where(keep, xs.abs(), torch.zeros_like(xs)) + (skip.double().abs() if with_skip else 0)
    fi = torch.finfo(DT[dtype])
    # the scale, the product and the sum round in fp32, the result to its type
    tol = 3 * U * mag + fi.eps / 2 * want.abs() * (1 + 4 * U) + fi.smallest_normal * fi.eps / 2
    y = G.lsam_dropout(x, p, seed, tick, layer=layer, k_offset=k0, skip=skip)
    close(y, want, tol)
    if not with_skip:
        assert torch.equal(y == 0, ~keep | (x == 0))
    # into a padded buffer whose padding stays, and in place
    buf = torch.full((K, rows, n + 5), 3.0, device="cuda", dtype=DT[dtype])
    G.lsam_dropout(x, p, seed, tick, layer=layer, k_offset=k0, skip=skip, out=buf[:, :, 2:2 + n])
    assert torch.equal(buf[:, :, 2:2 + n], y) and (buf[:, :, :2] == 3).all() and (buf[:, :, 2 + n:] == 3).all()
    x2 = x.clone(memory_format=torch.preserve_format)
    G.lsam_dropout(x2, p, seed, tick, layer=layer, k_offset=k0, skip=skip, out=x2)
    assert torch.equal(x2, y)


def test_dropout_mask_is_a_function_of_the_position_alone():
    ones = torch.ones((4, 40, 200), device="cuda")
    kw = dict(p=0.25, seed=3, tick=9, layer=2)
    full = G.lsam_dropout(ones, **kw)
    assert torch.equal(G.lsam_dropout(ones[1:3], k_offset=1, **kw), full[1:3])            # a shard of the workers
    assert torch.equal(G.lsam_dropout(ones[:, :7, :33], **kw), full[:, :7, :33])          # fewer rows, shorter rows
    assert torch.equal(G.lsam_dropout(ones.bfloat16(), **kw).float() > 0, full > 0)       # any type
    assert torch.equal(G.lsam_dropout(ones, **kw), full)                                  # the descent pass of the tick
    for other in (dict(kw, tick=10), dict(kw, tick=9 + (1 << 32)), dict(kw, layer=3), dict(kw, seed=4), dict(kw, seed=3 + (1 << 32))):
        diff = (G.lsam_dropout(ones, **other) > 0) != (full > 0)
        # two independent masks differ with probability 2 p (1 - p) = 0.375; 32000 positions, six standard deviations
        assert abs(diff.float().mean().item() - 0.375) < 6 * (0.375 * 0.625 / 32000) ** 0.5
    assert abs((full > 0).float().mean().item() - 0.75) < 6 * (0.75 * 0.25 / 32000) ** 0.5


def test_dropout_extremes():
    x = torch.randn((2, 3, 50), device="cuda")
    assert torch.equal(G.lsam_dropout(x, 0.0, 1, 1), x)
    assert torch.equal(G.lsam_dropout(x, 1.0, 1, 1), torch.zeros_like(x))
    assert torch.equal(G.lsam_dropout(x, 1.0, 1, 1, skip=x), x)
    y = G.lsam_dropout(torch.full_like(x, NAN), 0.5, 1, 1)
    assert torch.equal(torch.isnan(y), torch.from_numpy(keep_mask(2, 3, 50, 0.5, 1, 1, 0, 0)).cuda()) and (y.nan_to_num() == 0).all()
    assert G.lsam_dropout(x[:, :0], 0.5, 1, 1).shape == (2, 0, 50) and G.lsam_dropout(x[:, :, :0], 0.5, 1, 1).shape == (2, 3, 0)
    G.lsam_dropout(x, 0.5, (1 << 64) - 1, (1 << 64) - 1, layer=4095, k_offset=(1 << 20) - 2)


# ------------------------------------------------------------------------------------------------ refusals, streams, graphs, a run together
def test_refusals_on_the_device():
    l = torch.randn((1, 4, 100), device="cuda")
    y = torch.zeros((1, 4), device="cuda", dtype=torch.int32)
    r = G.lsam_logprob(l, y)
    bad = [
        lambda: G.lsam_logprob(l, y.long()), lambda: G.lsam_logprob(l, y[:, :3]), lambda: G.lsam_logprob(l, y.cpu()), lambda: G.lsam_logprob(l, y, top_k=33), lambda: G.lsam_logprob(l[:, :, :0], y),
        lambda: G.lsam_logprob_grad(l, y, r.lse, None), lambda: G.lsam_logprob_grad(l, None, r.lse, r.lse), lambda: G.lsam_logprob_grad(l, y, r.lse, None, dentropy=r.lse),
        lambda: G.lsam_logprob_grad(l, y, r.lse, r.lse, out=l[:, :1].expand(1, 4, 100)), lambda: G.lsam_logprob_grad(l, y, r.lse, r.lse, out=l.bfloat16()),
        lambda: G.lsam_head_logprob(l, l.bfloat16()), lambda: G.lsam_head_logprob(l, l[:, :, :50]), lambda: G.lsam_head_logprob(l, l.transpose(1, 2).contiguous().transpose(1, 2)),
        lambda: G.lsam_dropout(l.transpose(1, 2), 0.5, 1, 1), lambda: G.lsam_dropout(l, 0.5, 1, 1, skip=l[:, :2]), lambda: G.lsam_dropout(l, 2.0, 1, 1), lambda: G.lsam_dropout(l, 0.5, 1, 1, out=l[:, :1].expand(1, 4, 100)),
        lambda: G.lsam_dropout(l, 0.5, 1, 1, layer=1 << 32), lambda: G.lsam_dropout(l, 0.5, 1, 1, k_offset=1 << 32),  # would wrap in a 32-bit argument
        lambda: G.lsam_logprob_grad(l, y, r.lse, r.lse, out=torch.zeros(200, device="cuda").as_strided((1, 4, 100), (0, 3, 1))),
    ]
    for f in bad:
        with pytest.raises(G.LsamError) as e:
            f()
        assert e.value.code == G.LSAM_ERR_INVALID
    # host memory, pageable and pinned, and a misaligned address at the C boundary
    import ctypes as C

    err = C.create_string_buffer(256)
    for host in (torch.zeros(400), torch.zeros(400).pin_memory()):
        rc = G.lib().lsam_logprob(host.data_ptr(), 0, 1, 4, 100, 0, 100, 1, None, 0, None, r.lse.data_ptr(), None, None, None, None, err, 256)
        assert rc == G.LSAM_ERR_INVALID and b"device memory" in err.value
    rc = G.lib().lsam_logprob(l.data_ptr() + 2, 0, 1, 3, 100, 0, 100, 1, None, 0, None, r.lse.data_ptr(), None, None, None, None, err, 256)
    assert rc == G.LSAM_ERR_INVALID and b"aligned" in err.value
    torch.cuda.synchronize()


def test_side_streams_and_graphs():
    K, rows, C, D = 2, 64, 5000, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn((K, rows, D), generator=g, device="cuda").bfloat16()
    w = (torch.randn((K, C, D), generator=g, device="cuda") / 8).bfloat16()
    l = torch.randn((K, rows, C), generator=g, device="cuda").bfloat16()
    y = make_labels(K, rows, C, 0)

    def everything(stream=None):
        a = G.lsam_logprob(l, y, top_k=4, stream=stream)
        b = G.lsam_logprob_grad(l, y, a.lse, a.logp, stream=stream)
        c = G.lsam_head_logprob(h, w, y, stream=stream)
        d = G.lsam_dropout(h, 0.2, 1, 2, stream=stream)
        return [a.logp, a.lse, a.entropy, a.top_logp, a.top_idx, b, c.logp, c.lse, c.entropy, d]

    want = everything()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    both = [everything(s) for s in (s1, s2)]  # two at once
    with torch.cuda.stream(s1):
        both.append(everything())
    torch.cuda.synchronize()
    for got in both:
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = everything()
        graphs.append((gr, out))
    l2, h2, y2 = torch.randn_like(l), torch.randn_like(h), make_labels(K, rows, C, 5)
    l.copy_(l2); h.copy_(h2); y.copy_(y2)
    want = everything()
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        graphs[0][0].replay()
    with torch.cuda.stream(s2):
        graphs[1][0].replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_a_training_pass_of_them_together():
    # a residual block with dropout, a head, the cross-entropy with an entropy bonus, backward to the first weights: against 64-bit autograd
    K, B, D, C = 3, 50, 64, 37
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((K, B, D), generator=g, device="cuda")
    w1 = torch.randn((K, D, D), generator=g, device="cuda") / 8
    w2 = torch.randn((K, C, D), generator=g, device="cuda") / 8
    y = make_labels(K, B, C, 0)
    p, seed, tick, ent_w = 0.2, 99, 7, 0.05
    z = x @ w1.transpose(1, 2)
    act = torch.relu(z)
    h = G.lsam_dropout(act, p, seed, tick, skip=x)
    l = h @ w2.transpose(1, 2)
    sc = G.lsam_logprob(l, y)
    hs = G.lsam_head_logprob(h, w2, y)
    dl = G.lsam_logprob_grad(l, y, sc.lse, torch.full_like(sc.lse, -1.0 / B), entropy=sc.entropy, dentropy=torch.full_like(sc.lse, -ent_w / B))
    dw2 = dl.transpose(1, 2) @ h
    dh = dl @ w2
    dw1 = (G.lsam_dropout(dh, p, seed, tick) * (z > 0)).transpose(1, 2) @ x

    keep = torch.from_numpy(keep_mask(K, B, D, p, seed, tick, 0, 0)).cuda()
    cut = int(np.floor(p * 65536 + 0.5))
    a1, a2 = w1.double().requires_grad_(), w2.double().requires_grad_()
    hh = x.double() + torch.relu(x.double() @ a1.transpose(1, 2)) * keep * (65536 / (65536 - cut))
    lp = torch.log_softmax(hh @ a2.transpose(1, 2), -1)
    logp = lp.gather(-1, y.long().unsqueeze(-1)).squeeze(-1)
    ent = -(lp.exp() * lp).sum(-1)
    (-(logp.sum() + ent_w * ent.sum()) / B).backward()
    # fp32 products of 64 terms twice over, then sums over 50 samples: a few hundred roundings of 2^-24 at most, relative to the gradient's scale
    for got, want in ((dw1, a1.grad), (dw2, a2.grad)):
        assert (got - want).norm() / want.norm() < 400 * U
    assert (sc.logp - logp).abs().max() < 400 * U * 10 and (hs.logp - logp).abs().max() < 400 * U * 10
    assert (sc.entropy - ent).abs().max() < 400 * U * 10
