"""Refusals of prompt attention, rotated appending and logit adjustment: every one comes back before anything is enqueued, so no device is needed."""
import ctypes as C

import pytest

from paper_2507_06517_b200 import binding as B
from test_paged_host import BAD_SHAPES, F32, GOOD, P, lib, pool, table

BIG = 1 << 40
OUT = B._Tensor(4096, B.BF16, 8, 8, 8, 8)


def batch(layers=1, seqs=2, most=100, total=None, cu=None, ll=None, heads=0):
    return B._Batch(layers, seqs, most, seqs * most if total is None else total, cu, ll, heads)


def attend(keys=None, rows=None, hq=8, h=2, d=128, scale=0.0, q=GOOD, k=GOOD, v=GOOD, out=OUT, lse=None, ws=P, ws_bytes=BIG):
    return lib.spindlekv_prompt_attend(keys or batch(), rows, hq, h, d, scale, q, k, v, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(keys=batch(layers=0)), B.INVALID_ARG), (dict(keys=batch(seqs=0, total=100)), B.INVALID_ARG), (dict(keys=batch(most=0, total=0)), B.INVALID_ARG),
    (dict(keys=batch(total=150)), B.INVALID_ARG), (dict(keys=batch(cu=256, ll=256)), B.INVALID_ARG), (dict(rows=batch(seqs=3)), B.INVALID_ARG),
    (dict(rows=batch(layers=2)), B.INVALID_ARG), (dict(hq=0), B.INVALID_ARG), (dict(h=0), B.INVALID_ARG), (dict(hq=7), B.INVALID_ARG),
    (dict(d=96), B.UNSUPPORTED), (dict(d=256), B.UNSUPPORTED), (dict(hq=258, h=2), B.UNSUPPORTED), (dict(keys=batch(ll=256, heads=2)), B.UNSUPPORTED),
    (dict(keys=batch(layers=300, seqs=300)), B.UNSUPPORTED), (dict(hq=1025, h=1025), B.UNSUPPORTED), (dict(keys=batch(seqs=1, most=(1 << 30) + 1)), B.UNSUPPORTED)])
def test_prompt_attention_checks_its_shape(kw, want):
    assert attend(**kw) == want
    shape = {k: kw.get(k, v) for k, v in dict(keys=batch(), rows=None, hq=8, h=2, d=128).items()}
    assert lib.spindlekv_prompt_workspace_bytes(shape["keys"], shape["rows"], shape["hq"], shape["h"], shape["d"], B.BF16) == 0


def test_prompt_attention_checks_its_arguments():
    none = B._Tensor(None, B.BF16, 8, 8, 8, 8)
    odd = B._Tensor(264, B.BF16, 8, 8, 8, 8)
    bent = B._Tensor(256, B.BF16, 8, 8, 4, 8)
    for name in ("q", "k", "v", "out"):
        for t in (none, odd, bent, B._Tensor(256, 7, 8, 8, 8, 8)):
            assert attend(**{name: t}) == B.INVALID_ARG
    for name in ("k", "v"):
        assert attend(**{name: F32}) == B.UNSUPPORTED
    assert attend(out=B._Tensor(4096, B.F32, 8, 8, 8, 8)) == B.UNSUPPORTED
    assert attend(out=GOOD) == B.INVALID_ARG                                       # in place
    for scale in (-1.0, float("nan"), float("inf")):
        assert attend(scale=scale) == B.INVALID_ARG
    assert attend(lse=C.c_void_p(258)) == B.INVALID_ARG
    assert attend(ws=None) == B.INVALID_ARG and attend(ws=C.c_void_p(264)) == B.INVALID_ARG
    assert attend(ws_bytes=0) == B.WORKSPACE_TOO_SMALL
    assert lib.spindlekv_prompt_attend(None, None, 8, 2, 128, 0.0, GOOD, GOOD, GOOD, OUT, None, P, BIG, None) == B.INVALID_ARG
    # tensors that repeat memory
    flat = B._Tensor(8192, B.BF16, 0, 0, 8, 8)
    for name in ("q", "k", "v"):
        assert attend(**{name: flat}) == B.UNSUPPORTED
    assert attend(out=flat) == B.INVALID_ARG


def test_workspace_of_prompt_attention_covers_its_parts():
    def need(b, rows=None, hq=8, h=2, d=128, dtype=B.BF16):
        return lib.spindlekv_prompt_workspace_bytes(b, rows, hq, h, d, dtype)
    assert need(batch(seqs=8, most=4096)) == 256                                   # enough rows: no parts
    one = need(batch(seqs=1, most=16384), batch(seqs=1, most=1))
    assert one >= 256 + 2 * 8 * (128 * 4 + 8) and one < 1 << 20
    assert need(batch(seqs=1, most=16384), batch(seqs=1, most=1), dtype=B.F32) == one                               # few rows: nothing is taken apart
    assert need(batch(seqs=1, most=16384), batch(seqs=1, most=100), dtype=B.F32) >= 16384 * 2 * 2 * 128 * 6         # the pieces of every key and value


@pytest.mark.parametrize("p,t,want", BAD_SHAPES)
def test_rotated_append_checks_pool_and_table(p, t, want):
    none = B.NO_TENSOR
    assert lib.spindlekv_paged_append_rotated(pool(**p), table(**t), P, 1, GOOD, GOOD, 1, None, 0, 0, P, 10, None, none, 0, none, none, None) == want


def test_rotated_append_checks_its_arguments():
    pl, tb, none = pool(), table(), B.NO_TENSOR

    def call(start=P, new=4, K=GOOD, V=OUT, rows=4, idx=None, idx_len=0, idx_seq=0, rope=P, positions=100, first=None, K_out=none, hq=0, Q=none, Q_out=none):
        return lib.spindlekv_paged_append_rotated(pl, tb, start, new, K, V, rows, idx, idx_len, idx_seq, rope, positions, first, K_out, hq, Q, Q_out, None)

    moved = B._Tensor(256, B.BF16, 16, 8, 8, 8)
    for kw in (dict(start=None), dict(start=C.c_void_p(258)), dict(new=0), dict(rows=0), dict(K=none), dict(V=none), dict(rope=None), dict(rope=C.c_void_p(264)),
               dict(positions=0), dict(first=C.c_void_p(257)), dict(idx=P, idx_len=100, idx_seq=3), dict(idx=P, idx_len=11, idx_seq=4),
               dict(idx=P, idx_len=12, idx_seq=4, K_out=OUT), dict(idx=P, idx_len=12, idx_seq=4, hq=8, Q=GOOD, Q_out=OUT), dict(hq=-1), dict(hq=8), dict(hq=8, Q=GOOD),
               dict(K_out=moved), dict(hq=8, Q=GOOD, Q_out=moved), dict(K_out=B._Tensor(260, B.BF16, 8, 8, 8, 8)), dict(V=GOOD, K_out=GOOD), dict(K_out=B._Tensor(4096, B.BF16, 8, 0, 8, 8)), dict(hq=8, Q=GOOD, Q_out=B._Tensor(4096, B.BF16, 8, 8, 0, 8))):
        assert call(**kw) == B.INVALID_ARG, kw
    for kw in (dict(V=F32), dict(K_out=F32.__class__(4096, B.F32, 8, 8, 8, 8)), dict(hq=8, Q=F32, Q_out=B._Tensor(4096, B.F32, 8, 8, 8, 8)), dict(hq=70000, Q=GOOD, Q_out=OUT)):
        assert call(**kw) == B.UNSUPPORTED, kw


def test_logits_check_their_arguments():
    def call(n=4, v=100, logits=P, dtype=B.BF16, stride=100, out=C.c_void_p(4096), out_stride=100, rules=True, **kw):
        r = B._LogitRules()
        for k, x in kw.items():
            setattr(r, k, x)
        return lib.spindlekv_logits_adjust(n, v, logits, dtype, stride, r if rules else None, out, out_stride, None)

    for kw in (dict(n=0), dict(v=0), dict(logits=None), dict(out=None), dict(rules=False), dict(stride=-1), dict(dtype=2), dict(logits=C.c_void_p(257)),
               dict(dtype=B.F32, out=C.c_void_p(4098)), dict(out_stride=99), dict(out=P, out_stride=101), dict(history=256, max_history=-1), dict(history=256, history_stride=-1),
               dict(repetition=256), dict(presence=256), dict(frequency=256), dict(n_prompt=256), dict(history_lens=256), dict(n_bias=-1), dict(n_bias=2, bias_token=256),
               dict(n_bias=2, bias_value=256), dict(history=258, max_history=1), dict(allowed=257), dict(allowed=256, allowed_stride=-1), dict(history=256, max_history=1, repetition=257)):
        assert call(**kw) == B.INVALID_ARG, kw
    assert call(n=65536) == B.UNSUPPORTED
    assert call(v=(1 << 30) + 1, stride=1 << 31, out_stride=1 << 31) == B.UNSUPPORTED
