"""Refusals of the paged-cache and beam-selection calls: every one comes back before anything is enqueued, so no device is needed."""
import ctypes as C

import pytest

from paper_2507_06517_b200 import binding as B

lib = B._lib
P = C.c_void_p(256)                     # an aligned, non-null address that is never dereferenced
GOOD = B._Tensor(256, B.BF16, 8, 8, 8, 8)
F32 = B._Tensor(256, B.F32, 8, 8, 8, 8)


def pool(kc=256, vc=256, ks=256, vs=256, ref=256, n=64, ps=64, h=2, d=128, fmt=B.PAGED_INT8):
    return B._PagePool(kc, vc, ks, vs, ref, n, ps, h, d, fmt)


def table(pages=256, lens=512, layers=2, seqs=3, most=8):
    return B._PageTable(pages, lens, layers, seqs, most)


BAD_SHAPES = [(dict(kc=None), {}, B.INVALID_ARG), (dict(vc=264), {}, B.INVALID_ARG), (dict(ks=258), {}, B.INVALID_ARG), (dict(ref=None), {}, B.INVALID_ARG),
              (dict(n=0), {}, B.INVALID_ARG), (dict(n=(1 << 20) + 1), {}, B.UNSUPPORTED), (dict(ps=48), {}, B.UNSUPPORTED), (dict(ps=256), {}, B.UNSUPPORTED),
              (dict(h=0), {}, B.INVALID_ARG), (dict(d=96), {}, B.UNSUPPORTED), (dict(fmt=2), {}, B.UNSUPPORTED),
              ({}, dict(pages=None), B.INVALID_ARG), ({}, dict(lens=None), B.INVALID_ARG), ({}, dict(layers=0), B.INVALID_ARG),
              ({}, dict(most=0), B.INVALID_ARG), ({}, dict(layers=100, seqs=100), B.UNSUPPORTED), ({}, dict(most=1 << 25), B.UNSUPPORTED)]


@pytest.mark.parametrize("p,t,want", BAD_SHAPES)
def test_every_call_checks_pool_and_table(p, t, want):
    pl, tb = pool(**p), table(**t)
    big = 1 << 40
    assert lib.spindlekv_pages_workspace_bytes(pl, tb) == 0
    assert lib.spindlekv_paged_workspace_bytes(pl, tb, 8, 1) == 0
    assert lib.spindlekv_pages_resize(pl, tb, None, 1, P, P, big, None) == want
    assert lib.spindlekv_pages_fork(pl, tb, P, P, big, None) == want
    assert lib.spindlekv_pages_compact(pl, tb, P, P, big, None) == want
    assert lib.spindlekv_paged_append(pl, tb, P, 1, GOOD, GOOD, 1, None, 0, 0, None) == want
    assert lib.spindlekv_paged_attend(pl, tb, 8, 1, 100, 0.0, GOOD, GOOD, P, big, None) == want


def test_page_calls_check_their_arguments():
    pl, tb = pool(), table()
    need = lib.spindlekv_pages_workspace_bytes(pl, tb)
    assert need >= 64 * 4 + 2 * 3 * 8
    assert lib.spindlekv_pages_resize(None, tb, None, 1, P, P, need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_resize(pl, None, None, 1, P, P, need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_resize(pl, tb, None, 1, None, P, need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_resize(pl, tb, C.c_void_p(512), 1, P, P, need, None) == B.INVALID_ARG   # the lengths themselves
    assert lib.spindlekv_pages_resize(pl, tb, None, 1, P, C.c_void_p(260), need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_resize(pl, tb, None, 1, P, P, need - 1, None) == B.WORKSPACE_TOO_SMALL
    assert lib.spindlekv_pages_fork(pl, tb, None, P, need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_fork(pl, tb, P, P, need - 1, None) == B.WORKSPACE_TOO_SMALL
    assert lib.spindlekv_pages_fork(pl, table(layers=1, seqs=1025), P, P, 1 << 40, None) == B.UNSUPPORTED
    assert lib.spindlekv_pages_compact(pl, tb, None, P, need, None) == B.INVALID_ARG
    assert lib.spindlekv_pages_compact(pl, tb, P, None, need, None) == B.INVALID_ARG


def test_append_checks_its_arguments():
    def call(start=P, new=4, K=GOOD, V=GOOD, rows=4, idx=None, idx_len=0, idx_seq=0):
        return lib.spindlekv_paged_append(pool(), table(), start, new, K, V, rows, idx, idx_len, idx_seq, None)

    assert call(start=None) == B.INVALID_ARG
    assert call(new=0) == B.INVALID_ARG
    assert call(rows=0) == B.INVALID_ARG
    assert call(K=B._Tensor(264, B.BF16, 8, 8, 8, 8)) == B.INVALID_ARG
    assert call(V=B._Tensor(256, B.BF16, 8, 8, 8, 4)) == B.INVALID_ARG
    assert call(V=F32) == B.UNSUPPORTED
    assert call(idx=P, idx_len=12, idx_seq=3) == B.INVALID_ARG       # fewer than max_new entries per sequence
    assert call(idx=P, idx_len=11, idx_seq=4) == B.INVALID_ARG       # three sequences of four


def test_attend_checks_its_arguments():
    need = lib.spindlekv_paged_workspace_bytes(pool(), table(), 8, 1)
    assert need > 0

    def call(hq=8, rows=1, most=100, scale=0.0, q=GOOD, out=GOOD, ws=P, n=need):
        return lib.spindlekv_paged_attend(pool(), table(), hq, rows, most, scale, q, out, ws, n, None)

    assert call(hq=7) == B.INVALID_ARG
    assert call(hq=18) == B.UNSUPPORTED              # nine query heads per KV head
    assert call(rows=0) == B.INVALID_ARG
    assert call(rows=17) == B.UNSUPPORTED
    assert call(most=0) == B.INVALID_ARG
    assert call(scale=float("inf")) == B.INVALID_ARG
    assert call(scale=float("nan")) == B.INVALID_ARG
    assert call(q=B._Tensor(256, B.BF16, 8, 8, 8, 12)) == B.INVALID_ARG
    assert call(out=F32) == B.UNSUPPORTED
    assert call(ws=C.c_void_p(128)) == B.INVALID_ARG
    assert call(n=need - 1) == B.WORKSPACE_TOO_SMALL
    assert need == lib.spindlekv_paged_workspace_bytes(pool(), table(), 16, 16)      # one workspace serves every shape of a pool
    assert lib.spindlekv_paged_workspace_bytes(pool(), table(), 18, 1) == 0


def test_beam_checks_its_arguments():
    def call(n=2, w=4, v=100, k=4, logits=P, dtype=B.F32, stride=100, score=P, fin=None, eos=0, out=P, ws=P, nb=1 << 30):
        return lib.spindlekv_beam_select(n, w, v, k, logits, dtype, stride, score, fin, eos, out, P, P, ws, nb, None)

    assert call(n=0) == B.INVALID_ARG
    assert call(k=0) == B.INVALID_ARG
    assert call(w=1, v=3, k=4) == B.INVALID_ARG          # more than there are
    assert call(w=64, v=1 << 26) == B.INVALID_ARG        # positions beyond 31 bits
    assert call(w=65) == B.UNSUPPORTED
    assert call(k=33) == B.UNSUPPORTED
    assert call(n=40000) == B.UNSUPPORTED
    assert call(w=1, v=(1 << 30) + 1) == B.UNSUPPORTED
    assert call(logits=None) == B.INVALID_ARG
    assert call(logits=C.c_void_p(258)) == B.INVALID_ARG
    assert call(dtype=5) == B.INVALID_ARG
    assert call(stride=-1) == B.INVALID_ARG
    assert call(fin=P, eos=100) == B.INVALID_ARG
    assert call(out=None) == B.INVALID_ARG
    assert call(ws=C.c_void_p(8)) == B.INVALID_ARG
    assert call(nb=lib.spindlekv_beam_workspace_bytes(2, 4, 100, 4) - 1) == B.WORKSPACE_TOO_SMALL
    assert lib.spindlekv_beam_workspace_bytes(2, 65, 100, 4) == 0 and lib.spindlekv_beam_workspace_bytes(2, 4, 100, 33) == 0


def test_python_classes_refuse_what_does_not_fit():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)
    codes = z(4, 2, 32, 64, dt=torch.int8)
    sc, ref = z(4, 2, 2), z(4, dt=torch.int32)
    B.PagePool(codes, codes, sc, sc, ref)
    with pytest.raises(TypeError):
        B.PagePool(codes.float(), codes.float(), sc, sc, ref)
    with pytest.raises(TypeError):
        B.PagePool(codes, codes.view(torch.float8_e4m3fn), sc, sc, ref)
    with pytest.raises(ValueError):
        B.PagePool(codes, codes, sc[:, :, :1], sc, ref)
    with pytest.raises(ValueError):
        B.PagePool(codes.transpose(1, 2).contiguous().transpose(1, 2), codes, sc, sc, ref)
    with pytest.raises(ValueError):
        B.PageTable(z(1, 2, 3, dt=torch.int32), z(2, 1, dt=torch.int32))
    with pytest.raises(ValueError):
        B.PageTable(z(1, 2, 3), z(1, 2, dt=torch.int32))


def test_a_cache_owns_its_scratch_before_its_first_call():
    # made by a call, it would be filled on the current stream while the call's kernels run on another one
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache
    c = SpindleKVPagedCache(2, 3, 8, 2, 128, 64, 8, 64, device="cpu")
    for ws, need in ((c.ws_attend, lib.spindlekv_paged_workspace_bytes(c.pool.c, c.table.c, 8, 1)),
                     (c.ws_pages, lib.spindlekv_pages_workspace_bytes(c.pool.c, c.table.c))):
        assert ws is not None and ws.nbytes == need > 0 and not ws.any()


def test_the_hook_that_withholds_keys_can_be_set_and_restored():
    assert B.spindlekv_get_tuning(B.TUNE_PAGED_WITHHOLD) == -1
    try:
        B.spindlekv_set_tuning(B.TUNE_PAGED_WITHHOLD, 3)
        assert B.spindlekv_get_tuning(B.TUNE_PAGED_WITHHOLD) == 3
    finally:
        B.spindlekv_set_tuning(B.TUNE_PAGED_WITHHOLD, -1)
    assert B.spindlekv_get_tuning(B.TUNE_PAGED_WITHHOLD) == -1


def test_beam_refuses_scores_that_its_results_would_overwrite():
    # a sequence's results are written while others' scores are still read: only the same rows of the same buffer may be both
    def call(score, out, n=2, w=4, k=4):
        return lib.spindlekv_beam_select(n, w, 100, k, P, B.F32, 100, C.c_void_p(score), None, 0, C.c_void_p(out), P, P, P, 0, None)

    assert call(4096, 4096) == B.WORKSPACE_TOO_SMALL            # in place: all is well but the workspace given here
    for score, out, k in ((4096, 4100, 4), (4124, 4096, 4), (4096, 4096, 8), (4096, 4096, 2), (4096, 4124, 8), (4156, 4096, 8)):
        assert call(score, out, k=k) == B.INVALID_ARG
    for score, out, k in ((4096, 4128, 4), (4128, 4096, 4), (4160, 4096, 8)):
        assert call(score, out, k=k) == B.WORKSPACE_TOO_SMALL   # side by side
