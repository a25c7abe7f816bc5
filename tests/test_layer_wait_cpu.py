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
