"""Rotated appending refuses outputs that lie where another tensor of the call is read or written: before anything is enqueued, so no device is needed."""
import pytest

from paper_2507_06517_b200 import binding as B
from test_paged_host import P, lib, pool, table

AT = dict(K=256, V=4096, K_out=8192, Q=12288, Q_out=16384)


def call(at, hq=4):
    t = {n: B._Tensor(at[n], B.BF16, 8, 8, 8, 8) if at[n] else B.NO_TENSOR for n in AT}
    return lib.spindlekv_paged_append_rotated(pool(), table(), P, 4, t["K"], t["V"], 4, None, 0, 0, P, 100, None, t["K_out"], hq, t["Q"], t["Q_out"], None)


@pytest.mark.parametrize("out,where", [("K_out", "V"), ("K_out", "Q"), ("K_out", "Q_out"), ("Q_out", "K"), ("Q_out", "V")])
def test_outputs_lie_on_their_own_input_or_apart(out, where):
    assert call({**AT, out: AT[where]}) == B.INVALID_ARG


def test_outputs_lie_on_no_input_that_two_tensors_share():
    assert call({**AT, "V": AT["K"], "K_out": AT["K"]}) == B.INVALID_ARG              # in place, where the values are read too
    assert call({**AT, "Q": AT["K"], "K_out": AT["K"]}) == B.INVALID_ARG              # ... or the queries
    assert call({**AT, "Q": AT["K"], "Q_out": AT["K"]}) == B.INVALID_ARG
    assert call({**AT, "K_out": 0, "Q": AT["V"], "Q_out": AT["V"]}) == B.INVALID_ARG
    assert call({**AT, "Q": 0, "Q_out": 0, "K_out": AT["V"]}, hq=0) == B.INVALID_ARG
