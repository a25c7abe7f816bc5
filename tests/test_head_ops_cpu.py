"""Refusals of the operators around a classifier's head that need no GPU: every bad argument is turned into an error code on the host."""
import ctypes as C
import math
import random
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_2509_03110_b200 import binding as G

P = C.c_void_p(1 << 20)  # never dereferenced: each call below is refused before any pointer is used


def _call(fn, *args):
    err = C.create_string_buffer(256)
    rc = fn(*args, None, err, 256)
    return rc, err.value.decode()


def _logprob(dtype=0, K=1, rows=2, classes=5, sk=10, sr=5, sc=1, labels=P, top_k=0, logp=P):
    return _call(G.lib().lsam_logprob, P, dtype, K, rows, classes, sk, sr, sc, labels, top_k, logp, P, P, P, P)


def _grad(dtype=0, K=1, rows=2, classes=5, sk=10, sr=5, sc=1, labels=P, entropy=P, dlogp=P, dentropy=P, ok=10, orow=5, oc=1):
    return _call(G.lib().lsam_logprob_grad, P, dtype, K, rows, classes, sk, sr, sc, labels, P, entropy, dlogp, dentropy, P, ok, orow, oc)


def _head(dtype=1, K=1, rows=2, inner=8, classes=5, hr=8, wc=8, bk=0, labels=P, ws=P, nbytes=1 << 20):
    return _call(G.lib().lsam_head_logprob, P, P, None, dtype, K, rows, inner, classes, 16, hr, 40, wc, bk, labels, P, P, P, ws, nbytes)


def _dropout(dtype=0, K=1, rows=2, n=5, xr=5, orow=5, ok=10, p=0.5, layer=0, k_offset=0):
    return _call(G.lib().lsam_dropout, P, None, P, dtype, K, rows, n, 10, xr, 0, 0, ok, orow, p, 1, 2, layer, k_offset)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(K=-1), "K >= 0"), (dict(rows=-1), "rows >= 0"), (dict(classes=0), "classes"),
    (dict(classes=1 << 31), "classes"), (dict(top_k=-1), "top_k"), (dict(top_k=33), "top_k"), (dict(labels=None), "d_labels"),
    (dict(K=1 << 16, rows=1 << 16), "2^31"), (dict(sr=-5), "stride"), (dict(sk=1 << 62, K=3), "stride"), (dict(sr=1 << 61, rows=2), "stride")])
def test_logprob_refuses(kw, word):
    rc, msg = _logprob(**kw)
    assert rc == G.LSAM_ERR_INVALID and word in msg and msg.startswith("lsam_logprob: "), (rc, msg)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=7), "dtype"), (dict(classes=0), "classes"), (dict(dlogp=None, dentropy=None), "neither"), (dict(labels=None), "d_labels"), (dict(entropy=None), "d_entropy"),
    (dict(sc=-1), "stride"), (dict(orow=-1), "stride"), (dict(orow=0), "address"), (dict(oc=0), "address"), (dict(K=2, ok=0), "address"), (dict(orow=4), "address"), (dict(K=2, ok=9), "address"), (dict(K=2, ok=1, orow=5), "address"), (dict(K=1 << 16, rows=1 << 16), "2^31")])
def test_grad_refuses(kw, word):
    rc, msg = _grad(**kw)
    assert rc == G.LSAM_ERR_INVALID and word in msg, (rc, msg)


@pytest.mark.parametrize("kw, code, word", [
    (dict(dtype=5), G.LSAM_ERR_INVALID, "dtype"), (dict(inner=0), G.LSAM_ERR_INVALID, "inner"), (dict(classes=(1 << 30) + 1), G.LSAM_ERR_INVALID, "2^30"), (dict(inner=(1 << 30) + 1), G.LSAM_ERR_INVALID, "2^30"), (dict(classes=0), G.LSAM_ERR_INVALID, "classes"), (dict(labels=None), G.LSAM_ERR_INVALID, "d_labels"),
    (dict(K=65536), G.LSAM_ERR_INVALID, "65535"), (dict(rows=4194241), G.LSAM_ERR_INVALID, "4194240"), (dict(hr=-8), G.LSAM_ERR_INVALID, "stride"), (dict(bk=-1), G.LSAM_ERR_INVALID, "stride"), (dict(K=2, bk=1 << 61), G.LSAM_ERR_INVALID, "stride"),
    (dict(nbytes=4), G.LSAM_ERR_WORKSPACE, "workspace"), (dict(ws=C.c_void_p((1 << 20) + 16)), G.LSAM_ERR_WORKSPACE, "aligned")])
def test_head_refuses(kw, code, word):
    rc, msg = _head(**kw)
    assert rc == code and word in msg, (rc, msg)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "dtype"), (dict(p=-0.1), "p outside"), (dict(p=1.01), "p outside"), (dict(p=float("nan")), "p outside"), (dict(n=-1), "negative"), (dict(layer=-1), "layer"), (dict(layer=4096), "layer"),
    (dict(k_offset=-1), "workers"), (dict(k_offset=(1 << 20) - 1, K=2), "workers"), (dict(n=1 << 31), "2^31"), (dict(xr=-1), "stride"), (dict(orow=4), "address"), (dict(K=2, ok=0), "address"), (dict(K=2, ok=1), "address"), (dict(K=2, ok=7), "address"),
    (dict(rows=(1 << 31) - 1, n=(1 << 31) - 1, orow=(1 << 31) - 1, xr=0), "stride|2^31")])
def test_dropout_refuses(kw, word):
    rc, msg = _dropout(**kw)
    assert rc == G.LSAM_ERR_INVALID and any(w in msg for w in word.split("|")), (rc, msg)


def test_empty_calls_do_nothing():
    for kw in (dict(K=0), dict(rows=0)):
        assert _logprob(**kw)[0] == G.LSAM_OK and _grad(**kw)[0] == G.LSAM_OK and _head(**kw)[0] == G.LSAM_OK and _dropout(**kw)[0] == G.LSAM_OK
    assert _dropout(n=0)[0] == G.LSAM_OK


def test_host_pointers_are_refused():
    # without a GPU there is no current device; with one, these addresses are not device memory
    for call in (_logprob, _grad, _head, _dropout):
        rc, msg = call()
        assert rc == G.LSAM_ERR_INVALID and ("device" in msg or "pointer" in msg), msg


def test_error_buffer_is_optional():
    assert G.lib().lsam_dropout(P, None, P, 9, 1, 1, 1, 1, 1, 0, 0, 1, 1, 0.5, 1, 1, 0, 0, None, None, 0) == G.LSAM_ERR_INVALID


def test_workspace_bytes_grow_with_the_rows():
    f = G.lib().lsam_head_logprob_workspace_bytes
    assert f(1, 0, 1, 1, 1, 1) == 0 and f(1, 1, 0, 1, 1, 1) == 0 and f(1, 1, 1, 0, 1, 1) == 0 and f(1, 1, 1, 1, 0, 1) == 0 and f(3, 1, 1, 1, 1, 1) == 0 and f(1, 70000, 1, 1, 1, 1) == 0
    assert 0 < f(1, 1, 1, 64, 1, 1) <= f(1, 1, 4096, 64, 32768, 1) and f(1, 32, 256, 4096, 1000, 1) >= 32 * 256 * 16
    # what the tensor cores do not take as it is, is copied: 2 bytes an element, three planes for fp32, a shared head once
    copy = f(1, 4, 300, 1001, 5003, 0) - f(1, 4, 300, 1001, 5003, 1)
    assert copy >= 2 * 1008 * 4 * (300 + 5003) and f(0, 4, 300, 1001, 5003, 0) - f(1, 4, 300, 1001, 5003, 0) >= 4 * 1008 * 4 * (300 + 5003)
    assert f(1, 4, 300, 1001, 5003, 0) - f(1, 4, 300, 1001, 5003, 2) >= 2 * 1008 * 3 * 5003
    assert f(0, 1, 8, 4096, 32768, 1) < 1 << 20  # few rows are read where they are
    assert f(0, 1, 65535 * 32 + 1, 1, 1, 0) >= 3 * 2 * 8 * 65535 * 32  # more row tiles than a grid has: copied


def test_binding_refuses_what_is_not_a_cuda_tensor_of_the_right_form():
    x = torch.zeros(2, 8)
    for call in (lambda: G.lsam_logprob(x), lambda: G.lsam_dropout(x, 0.5, 1, 1), lambda: G.lsam_head_logprob(x, x), lambda: G.lsam_logprob_grad(x, None, None, None)):
        with pytest.raises(G.LsamError) as e:
            call()
        assert e.value.code == G.LSAM_ERR_INVALID
    for bad in (torch.zeros(8), torch.zeros(1, 2, 3, 4), torch.zeros(2, 8, dtype=torch.float64)):
        with pytest.raises(G.LsamError):
            G.lsam_logprob(bad)
    with pytest.raises(G.LsamError):
        G.lsam_dropout(x, 0.5, -1, 1)
    with pytest.raises(G.LsamError, match="workers"):  # would wrap in a 32-bit argument
        G.lsam_logprob(torch.zeros(1, 1, 1).expand(1 << 32, 1, 1))


def test_two_word_forms_refuse_as_the_others_do():
    for rc, msg in (_call(G.lib().lsam_logprob_wide, P, 3, 1, 2, 5, 10, 5, 1, P, 0, P, P, P, P, P, P),
                    _call(G.lib().lsam_logprob_wide, P, 0, 1, 2, 0, 10, 5, 1, P, 0, P, P, P, P, P, P)):
        assert rc == G.LSAM_ERR_INVALID and msg.startswith("lsam_logprob_wide: ")
    rc, msg = _call(G.lib().lsam_logprob_grad_wide, P, 0, 1, 2, 5, 10, 5, 1, P, P, P, P, None, None, P, 10, 5, 1)
    assert rc == G.LSAM_ERR_INVALID and msg.startswith("lsam_logprob_grad_wide: ") and "neither" in msg
    assert _call(G.lib().lsam_logprob_wide, P, 0, 0, 2, 5, 10, 5, 1, P, 0, P, P, P, P, P, P)[0] == G.LSAM_OK
    assert _call(G.lib().lsam_logprob_grad_wide, P, 0, 0, 2, 5, 10, 5, 1, P, P, P, P, P, P, P, 10, 5, 1)[0] == G.LSAM_OK


def _runs(K, rows, classes):
    """Runs of tiles per row tile by the whole search: falling widths, then falling runs, the first of equals."""
    pair = rows > 128
    ctas, m = (74, -(-rows // 256)) if pair else (148, -(-rows // 128))
    best = None
    for n in range(256, 31, -32 if pair else -16):
        tiles_n = -(-classes // n)
        for run in range(min(tiles_n, 32), 0, -1):
            runs = -(-tiles_n // run)
            tiles = float(-(-K * m * runs // ctas) * run)
            cost = (tiles * (n + 32) if pair else tiles * (n + 8) + 0.25 * n) * (1.0 + 0.02 / run)
            if best is None or cost < best[0]:
                best = cost, runs
    return best[1]


def test_the_plan_of_a_head_call_is_the_best_of_all_and_a_function_of_its_sizes():
    rng = random.Random(0)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    sizes = [(log(1, 64), log(1, 8192), log(1, 300000)) for _ in range(250)] + [(1, 4, 32768), (32, 256, 1000), (1, 4096, 32768), (1, 128, 1 << 30), (3, 129, 1)]
    f = G.lib().lsam_head_logprob_workspace_bytes
    up = lambda v: -(-v // 256) * 256  # noqa: E731
    want = [up(12 * 2 * _runs(*s) * s[0] * s[1]) + up(4 * s[0] * s[1]) for s in sizes]
    ask = lambda _: [f(G.BF16, K, rows, 64, classes, G.HEAD_ALIGNED) for K, rows, classes in sizes]  # noqa: E731
    assert ask(0) == want
    with ThreadPoolExecutor(4) as pool:
        assert all(got == want for got in pool.map(ask, range(8)))


def test_the_self_test_of_the_waits_refuses_as_the_call_does():
    f = G.lib().lsam_selftest_head_wait
    call = lambda dtype, K, rows, inner, classes: _call(f, P, P, dtype, K, rows, inner, classes, P, P, P, P, P, 1 << 20)  # noqa: E731
    for kw, word in (((5, 1, 2, 8, 5), "dtype"), ((1, 1, 2, 0, 5), "inner"), ((1, 1, 1 << 62, 8, 5), "rows"), ((1, 1, 2, 1 << 62, 5), "2^30"), ((1, 1, 2, 8, 1 << 62), "2^30"), ((0, 1, 2, 8, 5), "tensor cores")):
        rc, msg = call(*kw)
        assert rc == G.LSAM_ERR_INVALID and word in msg and msg.startswith("lsam_selftest_head_wait: "), (kw, msg)
    assert call(1, 0, 2, 8, 5)[0] == G.LSAM_OK
