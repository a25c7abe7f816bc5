"""Rows of no columns: what the C calls do without a GPU."""
from test_layer_ops_cpu import NONE, P, _norm, _norm_grad, _rows

from paper_2509_03110_b200 import binding as G


def test_the_gradient_of_a_gate_per_row_is_written_also_where_rows_have_no_columns():
    # a sum over no columns is zero, so the call has to reach its memory: a pointer of the host is refused, not passed over
    rc, msg = _norm_grad(n=0, gate=2, dz=_rows(P, 0, 0))
    assert rc == G.LSAM_ERR_INVALID and "device" in msg, (rc, msg)
    for kw in (dict(n=0, gate=2, dz=NONE), dict(n=0, rows=0, gate=2), dict(n=0, K=0, gate=2), dict(n=0, gate=1), dict(n=0, gate=3)):
        assert _norm_grad(**kw)[0] == G.LSAM_OK, kw
    assert _norm(n=0, gate=2)[0] == G.LSAM_OK
