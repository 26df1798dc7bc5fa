"""Rows that their positions rotate on the way into the 8-bit cache: bit for bit what rotating first and appending then gives."""
import numpy as np
import pytest
import torch

from paper_2507_06517_b200 import binding as B
from test_gpu_paged import DT, f64, fill, lens_t, make, ref_of, rows, same_state

pytestmark = pytest.mark.gpu


def table(n, d, base=10000.0):
    t = torch.empty((n, d // 2, 2), dtype=torch.float32, device="cuda")
    B.spindlekv_rope_table(d, n, base, t)
    return t


def turned(x, pos, rope):
    """Rows ``x`` ``[..., rows, d]`` at positions ``pos`` (broadcast over the rows' leading dimensions): fp32 numpy, each operation by itself, then x's type."""
    a, b = np.split(x.float().cpu().numpy(), 2, -1)
    p = np.broadcast_to(pos, a.shape[:-1])
    ok = (p >= 0) & (p < rope.shape[0])
    cs = rope.cpu().numpy()[np.where(ok, p, 0)]
    c, s = (np.where(ok[..., None], cs[..., i], np.float32("nan")).astype(np.float32) for i in (0, 1))
    with np.errstate(invalid="ignore"):
        return torch.from_numpy(np.concatenate([a * c - b * s, b * c + a * s], -1)).to(x.dtype)


def equal(got, want):
    return torch.equal(torch.nan_to_num(got.float().cpu(), nan=123456.0), torch.nan_to_num(want.float(), nan=123456.0))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,ps,hq", [(64, 16, 6), (128, 64, 11)])
def test_rows_and_queries_are_rotated_and_written(fmt, dtype, d, ps, hq):
    c = make(2, 4, None, 3, d, 60, 240 // ps, ps, fmt)
    rope = table(700, d)
    # nothing, one token, a block's end and beyond it; then on from there, into open blocks
    for step, lens in enumerate([[[0, 1, 15, 16], [17, 33, 47, 64]], [[1, 2, 16, 17], [17, 34, 90, 65]], [[2, 31, 51, 18], [81, 36, 101, 67]]]):
        r = ref_of(c)
        start = r.resize(np.array(lens))
        c.resize(lens_t(lens))
        n = int((np.array(lens) - start).max()) + (step == 1)
        K, V, Q = (rows((2, 4, h, n, d), dtype, 10 * step + i, 0.5 + step) for i, h in enumerate((3, 3, hq)))
        at = None if step == 0 else lens_t(np.array([[5, 0, 333, 100], [7, 8, 640, 695]]))
        first = start if at is None else at.cpu().numpy()
        pos = first[:, :, None, None] + np.arange(n)
        K_out, Q_out = torch.full_like(K, 9.0), torch.full_like(Q, 9.0)
        was = [x.clone() for x in (K, V, Q)]
        assert c.append_rotated(K, V, rope, first_pos=at, K_out=K_out, Q=Q, Q_out=Q_out) is Q_out
        assert c.status() == 0
        assert all(torch.equal(x, y) for x, y in zip((K, V, Q), was))
        new = (np.array(lens) - start)[:, :, None, None, None] > np.arange(n)[None, None, None, :, None]
        kk = turned(K, pos, rope)
        for got, want in ((K_out, kk), (Q_out, turned(Q, pos, rope))):
            assert equal(got, torch.where(torch.from_numpy(new), want, torch.full_like(want, 9.0)))
        r.append(start, f64(kk), f64(V))
        same_state(c, r)
        # in place, again: the same rows at the same places
        c.append_rotated(K, V, rope, first_pos=at, K_out=K, Q=Q, Q_out=Q)
        assert equal(K, torch.where(torch.from_numpy(new), kk, was[0].cpu())) and torch.equal(Q[..., :1, :] if n == 0 else Q, torch.where(torch.from_numpy(new).cuda(), Q_out, was[2]))
        same_state(c, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_by_list_keep_their_positions(dtype):
    d, h, n = 128, 2, 50
    for first in (None, [[3, 0, 100], [9, 9, 9]]):
        c = make(2, 3, None, h, d, 40, 4, 32, "int8")
        lens = [[50, 7, 0], [33, 16, 50]]
        r = ref_of(c)
        start = r.resize(np.array(lens))
        c.resize(lens_t(lens))
        rope = table(170, d)
        # token-major tensors with a gap behind every row; rows picked from 70 by lists with numbers outside
        K, V = (rows((2, 3, 70, h, 2 * d), dtype, s)[..., :d].transpose(2, 3) for s in (1, 2))
        idx = torch.randint(-3, 75, (2, h, 3 * n), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
        c.append_rotated(K, V, rope, idx=idx, first_pos=None if first is None else lens_t(first))
        pos = (0 if first is None else np.array(first))
        pos = np.broadcast_to(pos, (2, 3))[:, :, None, None] + np.arange(70)
        r.append(start, f64(turned(K, pos, rope)), f64(V), idx.cpu().numpy(), n)
        same_state(c, r)


def test_positions_outside_the_table_and_numbers_that_are_none():
    c = make(1, 4, None, 1, 64, 8, 2, 32, "int8")
    fill(c, [[20, 20, 20, 20]], "f32")
    r = ref_of(c)
    lens = [[30, 38, 21, 22]]
    start = r.resize(np.array(lens))
    c.resize(lens_t(lens))
    rope = table(25, 64)
    K, V = rows((1, 4, 1, 18, 64), "f32", 5), rows((1, 4, 1, 18, 64), "f32", 6)
    K[0, 3, 0, 1, 63] = float("inf")
    V[0, 2, 0, 0, 0] = float("nan")
    first = np.array([[20, -1, 3, 3]])                        # 20 .. 29: five of ten inside; -1: the first one is not
    K_out = torch.zeros_like(K)
    c.append_rotated(K, V, rope, first_pos=lens_t(first), K_out=K_out)
    kk = turned(K, first[:, :, None, None] + np.arange(18), rope)
    new = (np.array(lens) - start)[:, :, None, None, None] > np.arange(18)[None, None, None, :, None]
    assert equal(K_out, torch.where(torch.from_numpy(new), kk, torch.zeros_like(kk)))
    r.append(start, np.where(np.isfinite(f64(kk)), f64(kk), np.nan), np.where(np.isfinite(f64(V)), f64(V), np.nan))
    same_state(c, r)
    assert np.isnan(r.scale["k"]).sum() >= 3


def test_skipped_sequences_missing_pages_and_single_layers():
    c = make(2, 3, None, 2, 128, 30, 4, 32, "e4m3")
    r = fill(c, [[20, 33, 5], [40, 16, 64]], "bf16")
    rope = table(200, 128)
    K, V, Q = (rows((2, 3, h, 9, 128), "bf16", i) for i, h in enumerate((2, 2, 4)))
    K_out, Q_out = torch.full_like(K, 9.0), torch.full_like(Q, 9.0)
    c.append_rotated(K, V, rope, start=lens_t([[-1, 33, 9], [-1, -1, 70]]), K_out=K_out, Q=Q, Q_out=Q_out)       # start < 0 or >= lens
    assert (K_out == 9.0).all() and (Q_out == 9.0).all()
    same_state(c, r)
    # one layer of the two; its second sequence's page is not one of the pool: rows are turned, nothing is written
    c.pages[1, 1, 0] = 5000
    r.pages[1, 1, 0] = 5000
    start = np.array([[-1, -1, -1], [-1, 10, 60]])
    c.append_rotated(K[1:], V[1:], rope, start=lens_t(start), K_out=K_out[1:], Q=Q[1:], Q_out=Q_out[1:], layer=1)
    pos = start[1:, :, None, None] + np.arange(9)
    want = turned(K[1:], pos, rope)
    assert equal(K_out[1, 1, :, :6], want[0, 1, :, :6]) and (K_out[1, 1, :, 6:] == 9.0).all() and (K_out[0] == 9.0).all()
    assert equal(K_out[1, 2, :, :4], want[0, 2, :, :4])
    assert equal(Q_out[1, 1, :, :6], turned(Q[1:], pos, rope)[0, 1, :, :6]) and (Q_out[1, 0] == 9.0).all()
    kk = torch.zeros(K.shape)
    kk[1:] = want.float()
    r.append(np.array([[-1, -1, -1], [-1, -1, 60]]), f64(kk), f64(V))
    now = ref_of(c)
    for g in "kv":
        assert np.array_equal(now.codes[g], r.codes[g]) and np.array_equal(now.scale[g], r.scale[g], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_of_decoding_with_prompt_attention_logits_and_selection(dtype):
    """Prompt: rows rotated into the cache, attention over them; then a step: a rotated token, attention over the cache, adjusted logits, selected beams."""
    import prompt_ref as P
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect, SpindleKVLogits, SpindleKVPromptAttention, record_graph
    h, hq, d, n = 2, 4, 128, [70, 70, 70]
    c = make(1, 3, hq, h, d, 30, 8, 16, "int8")
    c.lens.zero_()
    rope = table(128, d)
    K, V, Q = (rows((1, 3, x, 70, d), dtype, i, 0.2) for i, x in enumerate((h, h, hq)))
    c.resize(lens_t([n]))
    c.append_rotated(K, V, rope, K_out=K, Q=Q, Q_out=Q)
    keys = B.Batch(1, 3, 70, 210)
    prompt = SpindleKVPromptAttention(keys, hq, h, d, DT[dtype])
    out = prompt.run(Q, K, V)
    want, _, bound = P.attend(Q, K, V, keys, keys)
    assert ((out.double() - want).abs() <= bound).all()
    # the cache's own attention of the last rows says the same, as far as 8 bits go
    last = c.attend(Q[:, :, :, -4:].contiguous())
    assert ((last.float() - out[:, :, :, -4:].float()).abs().max() / out.float().abs().max()) < 0.05
    k1, v1, q1 = (rows((1, 3, x, 1, d), dtype, 7 + i, 0.2) for i, x in enumerate((h, h, hq)))
    qr, got = torch.empty_like(q1), torch.empty_like(q1)
    adjust, select = SpindleKVLogits(3, 1000), SpindleKVBeamSelect(1, 3, 1000)
    logits = torch.randn((3, 1000), generator=torch.Generator().manual_seed(1)).to(DT[dtype]).cuda()
    history = torch.randint(0, 1000, (3, 70), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    z, score, two = torch.empty_like(logits), torch.zeros(3, device="cuda"), torch.full((3,), 2.0, device="cuda")

    def step():
        c.resize(add=1)
        c.append_rotated(k1, v1, rope, Q=q1, Q_out=qr)
        c.attend(qr, out=got)
        adjust.adjust(logits, out=z, history=history, repetition=two)
        return select.run(z, score)

    state = [t.clone() for t in (*c.pool.tensors, c.pages, c.lens)]
    first = [x.clone() for x in step()] + [got.clone(), qr.clone(), z.clone()]
    assert c.status() == 0
    for t, s in zip((*c.pool.tensors, c.pages, c.lens), state):
        t.copy_(s)
    graph = record_graph(step)
    for t, s in zip((*c.pool.tensors, c.pages, c.lens), state):
        t.copy_(s)
    for t in (got, qr, z):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    again = [select.score, select.parent, select.token, got, qr, z]
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert equal(qr, turned(q1, np.full((1, 3, 1, 1), 70), rope))


def test_offsets_beyond_32_bits():
    c, other = (make(2, 2, None, 2, 64, 20, 4, 32, "int8") for _ in range(2))
    rope, lens, gap = table(100, 64), [[40, 33], [50, 1]], 2576980480
    K, V, Q = (rows((2, 2, h, 50, 64), "bf16", i) for i, h in enumerate((2, 2, 4)))
    room = torch.empty(gap + 5 * Q[0].numel(), dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(room, t.shape, (gap, *t.stride()[1:]), i * Q[0].numel()) for i, t in enumerate((K, V, K, Q, Q))]
    for f, t in zip((far[0], far[1], far[3]), (K, V, Q)):
        f.copy_(t)
    outs = [torch.zeros_like(K), torch.zeros_like(Q)]
    far[2].zero_()
    far[4].zero_()
    for x in (c, other):
        x.resize(lens_t(lens))
    c.append_rotated(K, V, rope, K_out=outs[0], Q=Q, Q_out=outs[1])
    other.append_rotated(far[0], far[1], rope, K_out=far[2], Q=far[3], Q_out=far[4])
    assert torch.equal(far[2], outs[0]) and torch.equal(far[4], outs[1])
    same_state(other, ref_of(c))


def test_what_eviction_kept_is_rotated_on_the_way_into_the_cache():
    import gpu_util as U
    from paper_2507_06517_b200 import synth
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache, SpindleKVPass
    wl = synth.Workload("rotated", 3, 1, 8, 2, 128, "bf16", 32, (600, 600), 40, (0.05, 0.3), 4, "recency", budget_tokens=200.0, seed=13)
    host = U.generate(wl)
    p = SpindleKVPass(U.make_config(wl), wl.seq_lens, U.torch_dtype(wl))
    K, V = (U.stack_layers(wl, host, range(3), w) for w in "KV")
    p.evict(K[1:], V[1:], U.stack_layers(wl, host, [1, 2], "Q"))
    rope = table(600, 128)
    one, two = (SpindleKVPagedCache(2, 2, 8, 2, 128, 60, 12, 32, "int8") for _ in range(2))
    p.store_paged(K, V, one, rope_table=rope)
    whole = turned(K, np.arange(600), rope).cuda()
    p.store_paged(whole, V, two)
    assert one.status() == 0
    same_state(one, ref_of(two))


def test_refusals_of_the_class():
    c = make(1, 3, None, 2, 64, 20, 4, 32, "int8")
    rope = table(50, 64)
    K, V, Q = (rows((1, 3, h, 4, 64), "bf16", i) for i, h in enumerate((2, 2, 4)))
    for kw in (dict(K=K[:, :2]), dict(V=V[:, :, :, :3]), dict(K=K.float().cpu()), dict(rope_table=rope[..., 0]), dict(rope_table=rope.double()), dict(rope_table=table(50, 128)),
               dict(start=lens_t([[0, 0]])), dict(first_pos=torch.zeros((1, 3), device="cuda")), dict(Q=Q[:, :, :, :3]), dict(Q_out=Q), dict(K_out=K[:, :, :1]),
               dict(idx=torch.zeros((1, 3, 12), dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            c.append_rotated(**{"K": K, "V": V, "rope_table": rope, **kw})
    with pytest.raises(B.SpindleKVError):
        c.append_rotated(K, V, rope, idx=torch.zeros((1, 2, 12), dtype=torch.int32, device="cuda"), K_out=torch.empty_like(K))
    c.resize(lens_t([[4, 4, 4]]))
    made = c.append_rotated(K, V, rope, Q=Q)
    assert equal(made, turned(Q, np.arange(4), rope))
