"""Refusals of the self-tests of the waits that need no GPU."""
from test_layer_ops_cpu import BIG, P, _call, _res, _rows

from paper_2509_03110_b200 import binding as G


def _residual_wait(nbytes=BIG, **kw):
    n = kw.get("n", 8)
    row = lambda: _rows(P, 3 * n, n)  # noqa: E731
    return _call(G.lib().lsam_selftest_residual_wait, _res(branch=row(), gates=row(), **kw), row(), P, P, row(), row(), row(), row(), row(), P, P, P, nbytes)


def test_the_self_test_of_a_clusters_sums_refuses_as_the_call_does():
    for kw, word in ((dict(n=8), "cluster"), (dict(n=4096), "cluster"), (dict(n=32769), "cluster"), (dict(n=5000, dtype=1), "cluster"), (dict(n=5000, dtype=7), "dtype"), (dict(n=5000, act=9), "act"),
                     (dict(n=5000), "device")):
        rc, msg = _residual_wait(**kw)
        assert rc == G.LSAM_ERR_INVALID and word in msg and msg.startswith("lsam_selftest_residual_wait: "), (kw, msg)
    assert _residual_wait(n=5000, nbytes=64)[0] == G.LSAM_ERR_WORKSPACE


def test_the_self_test_of_the_products_refuses_as_the_call_does():
    f = G.lib().lsam_selftest_orthogonalize_wait
    call = lambda dtype=0, K=2, rows=100, cols=200, steps=5, a=3.4445, ws=P, nbytes=BIG: _call(  # noqa: E731
        f, P, dtype, K, rows, cols, rows * cols, cols, 1, steps, a, -4.775, 2.0315, 1.0, 1e-7, P, rows * cols, cols, 1, ws, nbytes)
    for kw, word in ((dict(dtype=1), "tensor cores"), (dict(rows=32), "tensor cores"), (dict(steps=0), "tensor cores"), (dict(dtype=4), "dtype"), (dict(steps=33), "steps"), (dict(a=0.5), "|a|"),
                     (dict(), "device")):
        rc, msg = call(**kw)
        assert rc == G.LSAM_ERR_INVALID and word in msg and msg.startswith("lsam_selftest_orthogonalize_wait: "), (kw, msg)
    assert call(nbytes=64)[0] == G.LSAM_ERR_WORKSPACE and call(K=0)[0] == G.LSAM_OK
