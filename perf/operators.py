"""Cases of the operators that stand around a classifier's head, with their plain forms.

Four operators: the log probabilities of given labels with log-sum-exp, entropy and the top alternatives of every row of
logits (`logprob`), the gradient of any loss of those two quantities with respect to the logits (`grad`), the same
quantities straight from activations and head weights without ever storing the logits (`head`), and dropout whose mask is
a counter-based function of (seed, tick, layer, worker, row, column) and is never stored (`dropout`).

`own = False` computes them with elementary torch operations in 32 bits, `own = True` calls the library's kernels.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
NEG_INF = float("-inf")


def listed():
    return [
        # one token of a large vocabulary: the latency of scoring a single position
        dict(name="logprob_token", op="logprob", K=1, rows=1, classes=32768, dtype="bf16", layout="row", pad=0, top_k=8, masked=False),
        # the classifier's own logits: 32 workers, minibatch 256, 1000 classes, stored with the sample index contiguous
        dict(name="logprob_workers", op="logprob", K=32, rows=256, classes=1000, dtype="fp32", layout="feature", pad=0, top_k=5, masked=False),
        # scoring a corpus against a large vocabulary
        dict(name="logprob_large", op="logprob", K=1, rows=2048, classes=131072, dtype="bf16", layout="row", pad=0, top_k=8, masked=False),
        # ragged batch: odd vocabulary, padded odd row stride, left-out and fully masked rows, masked classes
        dict(name="logprob_ragged", op="logprob", K=1, rows=777, classes=50021, dtype="fp16", layout="row", pad=4, top_k=20, masked=True),
        # training on the classifier's logits with an entropy term
        dict(name="grad_workers", op="grad", K=32, rows=256, classes=1000, dtype="fp32", layout="feature", pad=0, entropy=True, masked=False),
        # training on a large vocabulary
        dict(name="grad_large", op="grad", K=1, rows=2048, classes=131072, dtype="bf16", layout="row", pad=0, entropy=False, masked=False),
        # ragged batch of the training path
        dict(name="grad_ragged", op="grad", K=3, rows=211, classes=5003, dtype="fp16", layout="row", pad=2, entropy=True, masked=True),
        # scoring a sequence batch from its hidden states: a dense contraction
        dict(name="head_batch", op="head", K=1, rows=4096, inner=4096, classes=32768, dtype="bf16", bias=False, masked=False),
        # a few tokens against the whole head: the bytes of the head bound it
        dict(name="head_tokens", op="head", K=1, rows=4, inner=4096, classes=32768, dtype="bf16", bias=True, masked=False),
        # 32 workers, each with its own head of 1000 classes
        dict(name="head_workers", op="head", K=32, rows=256, inner=4096, classes=1000, dtype="bf16", bias=True, masked=True),
        # hidden activations of a residual layer of 32 workers on the way forward
        dict(name="dropout_forward", op="dropout", K=32, rows=256, n=4096, dtype="bf16", pad=0, skip=True),
        # the gradient of odd-sized padded fp32 activations on the way back
        dict(name="dropout_backward", op="dropout", K=7, rows=509, n=1021, dtype="fp32", pad=3, skip=False),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["logprob", "grad", "head", "dropout"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if op == "dropout":
        n = _log_int(rng, 1, 8192)
        rows = _log_int(rng, 1, min(8192, 32 * 1024 * 1024 // n))
        K = _log_int(rng, 1, max(1, min(32, 16 * 1024 * 1024 // (n * rows))))
        return dict(op=op, K=K, rows=rows, n=n, dtype=dtype, pad=rng.choice([0, 0, 1, 3, 8]), skip=rng.random() < 0.5)
    if op == "head":
        inner = _log_int(rng, 8, 4096) if dtype == "fp32" or rng.random() < 0.25 else 8 * _log_int(rng, 1, 512)
        classes = _log_int(rng, 2, 32768)
        most = (1 << 36) if dtype != "fp32" else (1 << 32)
        rows = _log_int(rng, 1, max(1, min(2048, most // (inner * classes))))
        K = _log_int(rng, 1, max(1, min(8, most // (inner * classes * rows))))
        return dict(op=op, K=K, rows=rows, inner=inner, classes=classes, dtype=dtype, bias=rng.random() < 0.5, masked=rng.random() < 0.5)
    classes = _log_int(rng, 1, 131072)
    rows = _log_int(rng, 1, max(1, min(8192, 64 * 1024 * 1024 // classes)))
    K = _log_int(rng, 1, max(1, min(32, 64 * 1024 * 1024 // (classes * rows))))
    case = dict(op=op, K=K, rows=rows, classes=classes, dtype=dtype, layout="feature" if classes <= 4096 and rng.random() < 0.5 else "row",
                pad=rng.choice([0, 0, 1, 4, 8]), masked=rng.random() < 0.5)
    if op == "logprob":
        case["top_k"] = rng.choice([0, 1, 5, 8, 20, 32])
    else:
        case["entropy"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    return g


def _labels(case, g, hidden_logits=None):
    """int32 labels [K, rows]; with `masked` one row in eight is left out (label -1)."""
    K, rows, classes = case["K"], case["rows"], case["classes"]
    y = torch.randint(0, classes, (K, rows), generator=g, device="cuda", dtype=torch.int32)
    if case["masked"]:
        out = torch.rand((K, rows), generator=g, device="cuda") < 0.125
        y = torch.where(out, torch.full_like(y, -1), y)
    return y


def _logits(case, g, y):
    """Logits [K, rows, classes] of the case's layout: normal, the label's raised by a few units as in a half-trained model.  With `masked`:
    a few classes of every row at -inf, one row in sixteen fully masked, garbage (NaN) in the rows that are left out."""
    K, rows, classes, pad = case["K"], case["rows"], case["classes"], case["pad"]
    dt = DTYPES[case["dtype"]]
    if case["layout"] == "feature":  # [K, classes, stride], the sample index contiguous
        view = torch.empty((K, classes, rows + pad), device="cuda", dtype=dt)[:, :, :rows].transpose(1, 2)
    else:
        view = torch.empty((K, rows, classes + pad), device="cuda", dtype=dt)[:, :, :classes]
    step = max(1, (1 << 27) // max(1, rows * classes))
    for k in range(0, K, step):  # whole workers at a time, for the memory of the 32-bit draw
        part = view[k:k + step]
        l = torch.randn(part.shape, generator=g, device="cuda") * 2.5
        yk = y[k:k + step].clamp(min=0).long().unsqueeze(-1)
        l.scatter_add_(-1, yk, torch.full(yk.shape, 4.0, device="cuda"))
        if case["masked"]:
            drop = torch.rand((classes,), generator=g, device="cuda") < 0.03
            l.masked_fill_(drop, NEG_INF)
            empty = torch.rand(part.shape[:2], generator=g, device="cuda") < 0.0625
            l.masked_fill_(empty.unsqueeze(-1), NEG_INF)
            l.masked_fill_((y[k:k + step] < 0).unsqueeze(-1), float("nan"))
        part.copy_(l)
    return view


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    s = dict(case=case)
    if op == "dropout":
        K, rows, n, pad = case["K"], case["rows"], case["n"], case["pad"]
        dt = DTYPES[case["dtype"]]
        draw_one = lambda: torch.randn((K, rows, n + pad), generator=g, device="cuda").to(dt)[:, :, :n]  # noqa: E731
        s["x"] = draw_one()
        s["skip"] = draw_one() if case["skip"] else None
        # what a training loop holds: its rate, its seed, the tick, the layer and the index of its first worker
        s.update(p=0.1 + 0.05 * (seed % 5), seed=(0x9E3779B97F4A7C15 * (seed + 1)) % (1 << 64), tick=(1 << 33) * (seed % 2) + 1000 + seed, layer=seed % 8, k_offset=3 * (seed % 4))
        return s
    if op == "head":
        K, rows, inner, classes = case["K"], case["rows"], case["inner"], case["classes"]
        dt = DTYPES[case["dtype"]]
        s["y"] = _labels(case, g)
        s["h"] = torch.randn((K, rows, inner), generator=g, device="cuda").to(dt)
        w = torch.empty((K, classes, inner), device="cuda", dtype=dt)
        for k in range(K):
            w[k].copy_(torch.randn((classes, inner), generator=g, device="cuda") * (2.0 / math.sqrt(inner)))
        s["w"] = w
        s["bias"] = 0.5 * torch.randn((K, classes), generator=g, device="cuda") if case["bias"] else None
        return s
    s["y"] = _labels(case, g)
    s["logits"] = _logits(case, g, s["y"])
    if op == "grad":
        # from the forward pass: log-sum-exp and entropy of every row; from the loss: the weights of the two
        K, rows, classes = case["K"], case["rows"], case["classes"]
        lse = torch.empty((K, rows), device="cuda")
        ent = torch.empty((K, rows), device="cuda")
        step = max(1, (1 << 26) // classes)
        for k in range(K):
            for r in range(0, rows, step):
                l = s["logits"][k, r:r + step].double()
                z = torch.logsumexp(l, -1)
                lp = l - z.unsqueeze(-1)
                p = lp.exp()
                lse[k, r:r + step] = z.float()
                ent[k, r:r + step] = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1).float()
        s["lse"], s["entropy"] = lse, ent
        s["dlogp"] = -(0.5 + torch.rand((K, rows), generator=g, device="cuda")) / rows
        s["dentropy"] = 0.01 * torch.randn((K, rows), generator=g, device="cuda") / rows if case["entropy"] else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_scores(l, y):
    """log probability of the label, log-sum-exp and entropy of the rows of l (32 bits); rows with a negative label are left out (0),
    rows with nothing but -inf have log-sum-exp -inf and entropy 0."""
    out = y < 0
    m = l.amax(-1, keepdim=True)
    e = torch.exp(l - torch.where(m == NEG_INF, torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    lse = torch.log(z) + torch.where(m == NEG_INF, torch.zeros_like(m), m)
    lp = l - lse
    ent = -torch.where(e == 0, torch.zeros_like(e), e * lp).sum(-1) / torch.where(z == 0, torch.ones_like(z), z).squeeze(-1)
    lse = lse.squeeze(-1)
    at = l.gather(-1, y.clamp(min=0).long().unsqueeze(-1)).squeeze(-1)
    logp = torch.where(at == NEG_INF, at, at - lse)
    zero = torch.zeros_like(lse)
    return torch.where(out, zero, logp), torch.where(out, zero, lse), torch.where(out, zero, ent)


def _plain_logprob(s):
    case, y = s["case"], s["y"]
    l = s["logits"].float()
    logp, lse, ent = _plain_scores(l, y)
    k = case["top_k"]
    if k == 0:
        return [logp, lse, ent]
    l = torch.where((y < 0).unsqueeze(-1), torch.full_like(l, NEG_INF), l)
    kk = min(k, case["classes"])
    v, i = torch.sort(l, dim=-1, descending=True, stable=True)
    v, i = v[..., :kk], i[..., :kk].to(torch.int32)
    gone = v == NEG_INF
    tv = torch.full((*y.shape, k), NEG_INF, device=l.device)
    ti = torch.full((*y.shape, k), -1, device=l.device, dtype=torch.int32)
    tv[..., :kk] = torch.where(gone, v, v - lse.unsqueeze(-1))
    ti[..., :kk] = torch.where(gone, torch.full_like(i, -1), i)
    return [logp, lse, ent, tv, ti]


def _plain_grad(s):
    l, y, lse = s["logits"].float(), s["y"], s["lse"]
    a = s["dlogp"].unsqueeze(-1)
    lp = l - lse.unsqueeze(-1)
    p = torch.exp(lp)
    g = -a * p
    g.scatter_add_(-1, y.clamp(min=0).long().unsqueeze(-1), a)
    if s["dentropy"] is not None:
        g = g - torch.where(p == 0, torch.zeros_like(p), p * (lp + s["entropy"].unsqueeze(-1))) * s["dentropy"].unsqueeze(-1)
    g = torch.where(((y < 0) | (lse == NEG_INF)).unsqueeze(-1), torch.zeros_like(g), g)
    return [g.to(s["logits"].dtype)]


def _plain_head(s):
    l = torch.matmul(s["h"].float(), s["w"].float().transpose(1, 2))
    if s["bias"] is not None:
        l = l + s["bias"].unsqueeze(1)
    return list(_plain_scores(l, s["y"]))


_M32 = 0xFFFFFFFF


def _plain_philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011) on int64 tensors that hold 32-bit words."""
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the low 64 bits of the products
        c0, c1, c2, c3 = (((b >> 32) & _M32) ^ c1 ^ k0), (b & _M32), (((a >> 32) & _M32) ^ c3 ^ k1), (a & _M32)
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return c0, c1, c2, c3


def _plain_dropout(s):
    x = s["x"]
    K, rows, n = x.shape
    dev = x.device
    i64 = lambda m: torch.arange(m, device=dev, dtype=torch.int64)  # noqa: E731
    group = i64((n + 7) // 8).view(1, 1, -1).expand(K, rows, -1)
    row = i64(rows).view(1, -1, 1).expand_as(group)
    word2 = (i64(K) + s["k_offset"] + (s["layer"] << 20)).view(-1, 1, 1).expand_as(group)
    tick, seed = s["tick"], s["seed"]
    w = _plain_philox(group, row, word2, torch.full_like(group, tick & _M32), (seed & _M32) ^ 0x64726F70, (seed >> 32) ^ (tick >> 32))
    bits = torch.stack([part for v in w for part in (v & 0xFFFF, v >> 16)], -1).reshape(K, rows, -1)[..., :n]
    dropped = int(math.floor(s["p"] * 65536 + 0.5))
    y = torch.where(bits >= dropped, x.float() * (65536.0 / (65536 - dropped)), torch.zeros((), device=dev))
    if s["skip"] is not None:
        y = y + s["skip"].float()
    return [y.to(x.dtype)]


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        from paper_2509_03110_b200 import binding as lsam

        if op == "logprob":
            r = lsam.lsam_logprob(s["logits"], s["y"], top_k=s["case"]["top_k"])
            return [r.logp, r.lse, r.entropy] + ([r.top_logp, r.top_idx] if s["case"]["top_k"] else [])
        if op == "grad":
            return [lsam.lsam_logprob_grad(s["logits"], s["y"], s["lse"], s["dlogp"], entropy=s["entropy"] if s["dentropy"] is not None else None, dentropy=s["dentropy"])]
        if op == "head":
            r = lsam.lsam_head_logprob(s["h"], s["w"], s["y"], bias=s["bias"])
            return [r.logp, r.lse, r.entropy]
        return [lsam.lsam_dropout(s["x"], s["p"], s["seed"], s["tick"], layer=s["layer"], k_offset=s["k_offset"], skip=s["skip"])]
    return {"logprob": _plain_logprob, "grad": _plain_grad, "head": _plain_head, "dropout": _plain_dropout}[op](s)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    size = 4 if case["dtype"] == "fp32" else 2
    rows = case["K"] * case["rows"]
    if op == "dropout":
        e = rows * case["n"]
        return {"bytes": e * size * (3 if case["skip"] else 2), "flops": e * (2 if case["skip"] else 1)}
    if op == "head":
        e = case["K"] * case["classes"]
        return {"bytes": size * (rows * case["inner"] + e * case["inner"]) + (4 * e if case["bias"] else 0) + 16 * rows,
                "flops": 2.0 * rows * case["inner"] * case["classes"] + 5.0 * rows * case["classes"]}
    live = rows * (0.875 if case["masked"] else 1.0)  # left-out rows are not read
    if op == "logprob":
        return {"bytes": live * case["classes"] * size + rows * (16 + 8 * case["top_k"]), "flops": 5.0 * live * case["classes"]}
    return {"bytes": live * case["classes"] * size + rows * case["classes"] * size + rows * (20 if case["entropy"] else 12), "flops": (6.0 if case["entropy"] else 4.0) * live * case["classes"]}


# ------------------------------------------------------------------------------------------------ 64 bits, from the definitions
def _exact_rows(l, y, top_k):
    """Scores of a [rows, classes] block in 64 bits: log softmax by sorting-free sums, entropy as -sum p log p, and the ranked alternatives."""
    left = y < 0
    l = l.masked_fill(left.unsqueeze(-1), 0.0)
    lse = torch.logsumexp(l, -1)
    empty = torch.isneginf(lse)
    lp = (l - lse.unsqueeze(-1)).masked_fill(empty.unsqueeze(-1), NEG_INF)
    ent = torch.special.entr(lp.exp()).sum(-1).masked_fill(empty, 0.0)
    logp = lp[torch.arange(len(y), device=y.device), y.clamp(min=0).long()]
    got = [logp.masked_fill(left, 0.0), lse.masked_fill(left, 0.0), ent.masked_fill(left, 0.0)]
    if top_k:
        kk = min(top_k, l.shape[-1])
        v, i = torch.sort(-lp, dim=-1, stable=True)
        v, i = -v[:, :kk], i[:, :kk]
        none = torch.isneginf(v) | left.unsqueeze(-1)
        tv = l.new_full((len(y), top_k), NEG_INF)
        ti = torch.full((len(y), top_k), -1, device=y.device, dtype=torch.int32)
        tv[:, :kk] = v.masked_fill(none, NEG_INF)
        ti[:, :kk] = i.int().masked_fill(none, -1)
        got += [tv, ti]
    return got


def _exact_dropout(s):
    x = s["x"].double().cpu().numpy()
    K, rows, n = x.shape
    groups = (n + 7) // 8
    m = np.uint64(0xFFFFFFFF)
    ctr = np.empty((4, K, rows, groups), np.uint64)
    ctr[0] = np.arange(groups, dtype=np.uint64)
    ctr[1] = np.arange(rows, dtype=np.uint64)[:, None]
    ctr[2] = (np.arange(K, dtype=np.uint64) + np.uint64(s["k_offset"] + s["layer"] * 1048576))[:, None, None]
    ctr[3] = np.uint64(s["tick"] % (1 << 32))
    key = [(s["seed"] % (1 << 32)) ^ 0x64726F70, (s["seed"] // (1 << 32)) ^ (s["tick"] // (1 << 32))]
    mul0, mul1, shift = np.uint64(0xD2511F53), np.uint64(0xCD9E8D57), np.uint64(32)
    for r in range(10):
        p0, p1 = ctr[0] * mul0, ctr[2] * mul1
        k0, k1 = np.uint64((key[0] + r * 0x9E3779B9) % (1 << 32)), np.uint64((key[1] + r * 0xBB67AE85) % (1 << 32))
        ctr = np.stack([(p1 >> shift) ^ ctr[1] ^ k0, p1 & m, (p0 >> shift) ^ ctr[3] ^ k1, p0 & m])
    words = np.ascontiguousarray(np.moveaxis(ctr, 0, -1).astype("<u4")).view("<u2").reshape(K, rows, groups * 8)[:, :, :n]
    cut = int(s["p"] * 65536 + 0.5)
    out = np.where(words.astype(np.int64) >= cut, x * 65536.0 / (65536 - cut), 0.0)
    if s["skip"] is not None:
        out = out + s["skip"].double().cpu().numpy()
    return [out]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        return _exact_dropout(s)
    K, rows, classes = case["K"], case["rows"], case["classes"]
    step = max(1, (1 << 26) // classes)
    parts = []
    for k in range(K):
        for r in range(0, rows, step):
            y = s["y"][k, r:r + step]
            if op == "head":
                l = s["h"][k, r:r + step].double() @ s["w"][k].double().T
                l = l if s["bias"] is None else l + s["bias"][k].double()
            else:
                l = s["logits"][k, r:r + step].double()
            if op != "grad":
                parts.append(_exact_rows(l, y, case.get("top_k", 0)))
                continue
            lse, a = s["lse"][k, r:r + step].double().unsqueeze(-1), s["dlogp"][k, r:r + step].double().unsqueeze(-1)
            p = torch.exp(l - lse)
            hot = (torch.arange(classes, device=l.device) == y.unsqueeze(-1)).double()
            g = a * (hot - p)
            if s["dentropy"] is not None:
                b, h = s["dentropy"][k, r:r + step].double().unsqueeze(-1), s["entropy"][k, r:r + step].double().unsqueeze(-1)
                g = g + b * (torch.special.entr(p) - h * p)
            parts.append([g.masked_fill((y < 0).unsqueeze(-1) | torch.isneginf(lse), 0.0)])
    cat = [torch.cat([p[j] for p in parts]) for j in range(len(parts[0]))]
    return [v.reshape(K, rows, *v.shape[1:]) for v in cat]
