"""Scoring a minibatch under the workers' iterates: against the loss the training step reports, a 64-bit forward pass, and an unscored twin run."""
import numpy as np
import pytest
import torch

from paper_2509_03110_b200 import binding as G
from paper_2509_03110_b200 import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

CONFIGS = {
    "mlp_fp32": dict(model=G.MODEL_MLP, widths=(40, 64, 33), K=3, batch=20),
    "mlp_fp32_narrow": dict(model=G.MODEL_MLP, widths=(40, 64, 10), K=2, batch=37),
    "resmlp_fp32": dict(model=G.MODEL_RESMLP, widths=(48, 64, 64, 20), K=2, batch=32),
    "mlp_planes": dict(model=G.MODEL_MLP, widths=(64, 128, 10), K=2, batch=64, gemm_impl=G.IMPL_TCGEN05),
    "mlp_planes_wide": dict(model=G.MODEL_MLP, widths=(64, 128, 40), K=2, batch=100, gemm_impl=G.IMPL_TCGEN05),
    "mlp_bf16": dict(model=G.MODEL_MLP, widths=(128, 256, 1000), K=4, batch=256, gemm_dtype=G.GEMM_BF16, gemm_impl=G.IMPL_TCGEN05),
    "resmlp_bf16_narrow": dict(model=G.MODEL_RESMLP, widths=(128, 128, 128, 10), K=2, batch=70, gemm_dtype=G.GEMM_BF16, gemm_impl=G.IMPL_TCGEN05),
    "mlp_bf16_simt": dict(model=G.MODEL_MLP, widths=(50, 64, 12), K=2, batch=33, gemm_dtype=G.GEMM_BF16, gemm_impl=G.IMPL_SIMT),
    "cnn": dict(model=G.MODEL_CNN, widths=(3, 8, 24, 10), K=2, batch=16, n_conv=1, img_h=8, img_w=8),
    "cnn_bf16_wide": dict(model=G.MODEL_CNN, widths=(3, 8, 24, 30), K=2, batch=16, n_conv=1, img_h=8, img_w=8, gemm_dtype=G.GEMM_BF16),
    "async": dict(model=G.MODEL_MLP, widths=(40, 64, 20), K=6, batch=16, active_num=100, tau=64),
    "async_bf16": dict(model=G.MODEL_MLP, widths=(64, 128, 20), K=6, batch=64, active_num=100, tau=64, gemm_dtype=G.GEMM_BF16, gemm_impl=G.IMPL_TCGEN05),
}


def make(cfg, seed=0, **more):
    c = dict(cfg, **more)
    n_in = c["widths"][0] * c.get("img_h", 1) * c.get("img_w", 1)
    classes = c["widths"][-1]
    X, labels = synth.gaussian_mixture(256, n_in, classes, seed=seed)
    gcfg = G.make_config(c.pop("model"), widths=c.pop("widths"), n_samples=256, lam=0.1, seed=3, **dict(dict(tau=8), **c))
    rng = np.random.default_rng(seed)
    d = G.lsam_param_count(gcfg)
    assert d > 0
    x0 = (rng.standard_normal((gcfg.K, d)) * 0.08).astype(np.float32)
    dX, dY = torch.from_numpy(X.astype(np.float32)).cuda(), torch.from_numpy(labels.astype(np.int32)).cuda()
    stream = torch.cuda.Stream() if gcfg.flags & G.FLAG_CUDA_GRAPH else None
    torch.cuda.synchronize()
    ctx = G.Lsam(gcfg, dX, dY, torch.from_numpy(x0).cuda(), torch.from_numpy(x0.mean(0)).cuda(), stream=stream)
    xb = rng.standard_normal((gcfg.K, gcfg.batch, n_in)).astype(np.float32)
    yb = rng.integers(0, classes, (gcfg.K, gcfg.batch)).astype(np.int32)
    return ctx, xb, yb, classes


@pytest.mark.parametrize("name", CONFIGS)
def test_scores_give_the_loss_of_the_training_step(name):
    ctx, xb, yb, C = make(CONFIGS[name])
    for _ in range(3):
        ctx.step(0.02, 0.05)
    k = min(5, C)
    r = ctx.score_batch(xb, yb, top_k=k)
    dev = ctx.score_batch(torch.from_numpy(xb).cuda(), torch.from_numpy(yb).cuda(), top_k=k)  # the same arrays on the device
    assert all(torch.equal(a, b) for a, b in zip(r, dev))
    loss = np.zeros(ctx.K, np.float32)
    ctx.step_batch(0.02, 0.05, xb, yb, h_loss=loss)
    torch.cuda.synchronize()
    stepped = ctx.read_active().astype(bool)
    assert stepped.any()
    lse = r.lse.abs().max().item()
    # the same fp32 logits, summed in another order: C / 8 terms in sequence at most, the exponential, the logarithm and the mean
    tol = 2 * ((C / 8 + 72) * U + 4 * U * (1 + lse)) + U * np.abs(loss)
    got = -r.logp.double().mean(1).cpu().numpy()
    assert (np.abs(got - loss) <= tol)[stepped].all(), (got, loss, tol)
    # the alternatives are the classes of largest probability, and the label's is among them where its logp says so
    p = r.top_logp.double().exp()
    assert (r.top_logp[..., :-1] >= r.top_logp[..., 1:]).all() and (p.sum(-1) <= 1 + 1e-5).all()
    hit = r.top_idx == torch.from_numpy(yb).cuda().unsqueeze(-1)
    at = (r.top_logp * hit).sum(-1)
    assert torch.equal(at[hit.any(-1)], r.logp[hit.any(-1)])
    assert ctx.status() == 0
    ctx.close()


@pytest.mark.parametrize("name", ["mlp_fp32", "mlp_fp32_narrow"])
def test_scores_against_a_64_bit_forward_pass(name):
    ctx, xb, yb, C = make(CONFIGS[name])
    ctx.step(0.02, 0.05)
    yb[0, 0] = -1  # left out
    r = ctx.score_batch(xb, yb)
    D, H = ctx.cfg.widths[0], ctx.cfg.widths[1]
    for k in range(ctx.K):
        v = torch.from_numpy(ctx.read_params(k)).double()
        W1, b1, W2, b2 = v[:D * H].view(H, D), v[D * H:D * H + H], v[D * H + H:D * H + H + H * C].view(C, H), v[-C:]
        x = torch.from_numpy(xb[k]).double()
        h = torch.relu(x @ W1.T + b1)
        l = h @ W2.T + b2
        # fp32 accumulation of D (H) products and one bias; the first layer's error passes through |W2|
        e1 = (D + 2) * U * (x.abs() @ W1.abs().T + b1.abs())
        el = e1 @ W2.abs().T + (H + 2) * U * (h.abs() @ W2.abs().T + b2.abs())
        lse = torch.logsumexp(l, -1)
        tol = 2 * el.amax(-1) + (C / 8 + 72) * U + 4 * U * (1 + lse.abs())
        want = l.gather(1, torch.from_numpy(yb[k]).clamp(min=0).long()[:, None])[:, 0] - lse
        live = torch.from_numpy(yb[k] >= 0)
        assert ((r.logp[k].cpu().double() - want).abs() <= tol)[live].all()
        assert ((r.lse[k].cpu().double() - lse).abs() <= tol)[live].all()
    assert r.logp[0, 0] == 0 and r.lse[0, 0] == 0 and r.entropy[0, 0] == 0
    assert ctx.status() == 0  # a left-out label is no bad index
    ctx.close()


@pytest.mark.parametrize("name, more", [("mlp_fp32", {}), ("mlp_planes", {}), ("mlp_bf16", {}), ("cnn", {}), ("async", {}), ("async_bf16", {}),
                                        ("mlp_fp32_narrow", dict(flags=G.FLAG_CUDA_GRAPH)), ("mlp_bf16", dict(flags=G.FLAG_CUDA_GRAPH | G.FLAG_PDL))])
def test_a_run_with_scoring_is_the_run_without(name, more):
    a, xb, yb, _ = make(CONFIGS[name], **more)
    b, _, _, _ = make(CONFIGS[name], **more)
    for t in range(6):
        a.score_batch(xb, yb, top_k=3)
        for c in (a, b):
            c.step(0.02, 0.05)
        assert np.array_equal(a.read_active(), b.read_active())
        first = a.score_batch(xb, yb, top_k=3)
        assert np.array_equal(a.read_active(), b.read_active())  # the mask of the last tick is put back
    again = a.score_batch(xb, yb, top_k=3)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    assert np.array_equal(a.read_all_params(), b.read_all_params())
    assert all(np.array_equal(p, q) for p, q in zip(a.read_step_info(), b.read_step_info()))
    a.close()
    b.close()


def test_scoring_refusals():
    ctx, xb, yb, C = make(CONFIGS["mlp_fp32"])
    for f in (lambda: ctx.score_batch(xb[:, :5], yb), lambda: ctx.score_batch(xb, yb.astype(np.int64)), lambda: ctx.score_batch(xb[:, :, :7].copy(), yb),
              lambda: ctx.score_batch(torch.from_numpy(xb).cuda(), yb), lambda: ctx.score_batch(xb, yb, top_k=33)):
        with pytest.raises(G.LsamError) as e:
            f()
        assert e.value.code == G.LSAM_ERR_INVALID
    out = torch.zeros(xb.shape[:2], device="cuda")
    L = G.lib()
    ptr = lambda a: G.C.c_void_p(a.ctypes.data if isinstance(a, np.ndarray) else a.data_ptr())  # noqa: E731
    assert L.lsam_score_batch(ctx._h, ptr(xb), None, 1, 0, ptr(out), None, None, None, None) == G.LSAM_ERR_INVALID        # logp without labels
    assert L.lsam_score_batch(ctx._h, ptr(xb), None, 1, 3, None, ptr(out), None, None, None) == G.LSAM_ERR_INVALID        # alternatives without arrays
    assert L.lsam_score_batch(ctx._h, None, None, 1, 0, None, ptr(out), None, None, None) == G.LSAM_ERR_INVALID
    assert L.lsam_score_batch(None, ptr(xb), None, 1, 0, None, ptr(out), None, None, None) == G.LSAM_ERR_INVALID
    assert L.lsam_score_batch(ctx._h, ptr(xb), None, 1, 0, None, ptr(xb), None, None, None) == G.LSAM_ERR_INVALID         # a result in host memory
    assert "lsam_logprob" in ctx.last_error()
    ctx.stage_batch(xb, yb)
    with pytest.raises(G.LsamError) as e:
        ctx.score_batch(xb, yb)
    assert e.value.code == G.LSAM_ERR_STATE
    ctx.step_staged(0.02, 0.05)
    assert ctx.score_batch(xb).logp is None
    ctx.close()
    flat = G.Lsam(G.make_config(G.MODEL_FLAT, K=2, flat_d=64), None, None, torch.zeros(2, 64, device="cuda"), torch.zeros(64, device="cuda"))
    assert L.lsam_score_batch(flat._h, ptr(xb), None, 1, 0, None, ptr(out), None, None, None) == G.LSAM_ERR_INVALID
    flat.close()
