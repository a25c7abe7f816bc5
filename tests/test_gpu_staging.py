"""The prefetch queue beside the other calls that take a minibatch: whatever is in flight, every tick trains on its own."""
import numpy as np
import pytest
import torch

from paper_2509_03110_b200 import binding as G
from test_gpu_score_batch import CONFIGS, make

pytestmark = pytest.mark.gpu

NAMES = ["mlp_fp32", "mlp_planes", "mlp_bf16", "cnn"]


def batches(ctx, n, classes, on_device):
    """n minibatches [K, B, in], pinned or on the device."""
    rng = np.random.default_rng(n)
    n_in = ctx.cfg.widths[0] * (ctx.cfg.img_h * ctx.cfg.img_w if ctx.cfg.model == G.MODEL_CNN else 1)
    out = [(torch.from_numpy(rng.standard_normal((ctx.K, ctx.cfg.batch, n_in)).astype(np.float32)),
            torch.from_numpy(rng.integers(0, classes, (ctx.K, ctx.cfg.batch)).astype(np.int32))) for _ in range(n)]
    out = [tuple(t.cuda() if on_device else t.pin_memory() for t in b) for b in out]
    torch.cuda.synchronize()  # the copy stream does not wait for what produced a device source
    return out


def busy(ctx, ms=20):
    """Work in front of whatever the context's stream gets next."""
    with torch.cuda.stream(ctx.stream):
        torch.cuda._sleep(int(ms * 1.9e6))


def same(a, b):
    torch.cuda.synchronize()
    assert a.status() == 0 and b.status() == 0
    assert np.array_equal(a.read_all_params(), b.read_all_params())
    a.close()
    b.close()


@pytest.mark.parametrize("on_device", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_a_minibatch_staged_behind_a_score_is_the_one_trained_on(name, on_device):
    a, _, _, C = make(CONFIGS[name], tau=64)
    b, _, _, _ = make(CONFIGS[name], tau=64)
    for s, x in zip(batches(a, 4, C, on_device), batches(a, 5, C, on_device)):  # one staged minibatch a round: both slots take their turn
        for c in (a, b):
            c.step(0.02, 0.05)
        quiet = a.score_batch(*s, top_k=3)
        torch.cuda.synchronize()
        busy(a)
        scores = a.score_batch(*s, top_k=3)
        for c in (a, b):
            c.stage_batch(*x)
            c.step_staged(0.02, 0.05)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(scores, quiet))
    same(a, b)


@pytest.mark.parametrize("on_device", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_a_supplied_minibatch_beside_staged_ones(name, on_device):
    a, _, _, C = make(CONFIGS[name], tau=64)
    b, _, _, _ = make(CONFIGS[name], tau=64)
    x = batches(a, 4, C, on_device)
    for c in (a, b):
        c.step(0.02, 0.05)
    for rounds in range(2):  # the queue starts at slot 0, then at slot 1
        # none, one and two minibatches wait while another one is trained on; then one is staged behind a tick that has not begun
        a.stage_batch(*x[0])
        a.step_batch(0.02, 0.05, *x[1])
        a.stage_batch(*x[2])
        a.step_batch(0.02, 0.05, *x[3])
        a.step_staged(0.02, 0.05)
        a.step_staged(0.02, 0.05)
        busy(a)
        a.step_batch(0.02, 0.05, *x[0])
        a.stage_batch(*x[3])
        a.step_staged(0.02, 0.05)
        for i in (1, 3, 0, 2, 0, 3):
            b.step_batch(0.02, 0.05, *x[i])
    same(a, b)


class Unsynchronised(torch.cuda.Stream):
    """A stream on which the binding's wait after lsam_init does nothing, as for a caller of the C interface that does not wait."""

    def synchronize(self):
        pass


def test_a_minibatch_staged_right_after_init_is_not_cleared_with_the_workspace():
    rng = np.random.default_rng(0)
    cfg = G.make_config(G.MODEL_MLP, widths=(40, 64, 10), K=2, batch=16, n_samples=64, tau=64, lam=0.1, seed=3)
    d = G.lsam_param_count(cfg)
    x0 = torch.from_numpy((rng.standard_normal((2, d)) * 0.08).astype(np.float32)).cuda()
    X, Y, y0 = torch.zeros((64, 40), device="cuda"), torch.zeros(64, device="cuda", dtype=torch.int32), x0.mean(0)
    xb, yb = torch.randn((2, 16, 40), device="cuda"), torch.randint(0, 10, (2, 16), device="cuda", dtype=torch.int32)
    runs = []
    for _ in range(2):
        stream = Unsynchronised()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(int(20 * 1.9e6))
        ctx = G.Lsam(cfg, X, Y, x0, y0, stream=stream)
        if runs:
            torch.cuda.synchronize()
        ctx.stage_batch(xb, yb)
        ctx.step_staged(0.02, 0.05)
        torch.cuda.synchronize()
        runs.append((ctx, ctx.read_all_params()))
    assert np.array_equal(runs[0][1], runs[1][1])
    for ctx, _ in runs:
        ctx.close()


def test_a_staged_copy_has_ended_when_the_context_has():
    K, B, n = 16, 512, 4096  # 134 MB: a few milliseconds from pinned memory
    cfg = G.make_config(G.MODEL_LSQ, widths=(n,), K=K, batch=B, n_samples=64, tau=64, lam=0.1, seed=3)
    x0 = torch.zeros((K, G.lsam_param_count(cfg)), device="cuda")
    ctx = G.Lsam(cfg, torch.zeros((64, n), device="cuda"), torch.zeros(64, device="cuda"), x0, x0[0].clone())
    xb, yb = torch.full((K, B, n), 3.0).pin_memory(), torch.zeros((K, B)).pin_memory()
    at, nbytes = ctx.workspace.data_ptr(), ctx.workspace.numel()
    ctx.stage_batch(xb, yb)
    ctx.close()
    del ctx
    z = torch.full((nbytes,), 7, dtype=torch.uint8, device="cuda")
    assert z.data_ptr() == at  # the workspace's memory
    torch.cuda.synchronize()
    assert (z == 7).all()
