"""Beam search's selection on the GPU against float64: parents and tokens exactly, scores to fp32."""
import numpy as np
import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu


def run(logits, score, n_beams, n_out, finished=None, eos=0):
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect
    n = logits.shape[0] // n_beams
    sel = SpindleKVBeamSelect(n, n_beams, logits.shape[1], n_out)
    out = sel.run(logits, score, finished=finished, eos=eos)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in out]


def check(logits, score, n_beams, n_out, finished=None, eos=0):
    got = run(logits, score, n_beams, n_out, finished, eos)
    want = R.beam(logits.double().cpu().numpy(), score.double().cpu().numpy(), n_beams, n_out, None if finished is None else finished.cpu().numpy(), eos)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    # the score: half an fp32 step of its own, and the exp-sum's relative error: 2^-22 per power and 40 roundings of 2^-24
    fin = np.isfinite(want[0])
    assert np.array_equal(got[0][~fin], want[0][~fin])
    assert (np.abs(got[0] - want[0])[fin] <= 2.0 ** -24 * np.abs(want[0][fin]) + 2.0 ** -22 + 40 * 2.0 ** -24).all()


def logits_of(rows, vocab, dtype, seed, spread=2.5):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, vocab), generator=gen) * spread).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,w,vocab,k", [(1, 1, 1, 1), (1, 1, 5, 5), (3, 4, 2, 8), (2, 4, 32000, 4), (1, 8, 2048, 16), (2, 3, 8193, 32), (5, 16, 50257, 16),
                                         (1, 64, 777, 32), (40, 8, 9001, 8), (1, 1, 128256, 32)])
def test_selection(dtype, n, w, vocab, k):
    check(logits_of(n * w, vocab, dtype, vocab + k), -torch.rand(n * w, generator=torch.Generator().manual_seed(1)).cuda() * 3, w, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_index(dtype):
    # three values only, equal beams, all equal, and zeros of both signs
    gen = torch.Generator().manual_seed(4)
    x = torch.randint(0, 3, (8, 20000), generator=gen).to(dtype).cuda()
    x[1] = x[0]
    check(x, torch.zeros(8, device="cuda"), 4, 32)
    check(torch.zeros((6, 9000), dtype=dtype, device="cuda"), torch.zeros(6, device="cuda"), 3, 17)
    z = torch.zeros((2, 5000), dtype=dtype, device="cuda")
    z[:, ::2] = -0.0
    check(z, torch.zeros(2, device="cuda"), 2, 9)


def test_order_and_reverse_order():
    # the largest logits all in one thread's, one slice's or the last slice's elements
    up = torch.linspace(-5, 5, 40000).repeat(4, 1).cuda()
    up += torch.arange(4, device="cuda")[:, None] * 1e-3
    s = torch.tensor([-1.0, -1.1, -1.2, -1.3], device="cuda")
    check(up, s, 2, 32)
    check(up.flip(1).contiguous(), s, 4, 32)


def test_masked_tokens_dead_beams_and_bad_rows():
    x = logits_of(12, 3000, torch.float32, 7)
    x[0, 3:] = -float("inf")                  # three tokens left
    x[1] = -float("inf")                      # none
    x[2, 100] = float("nan")
    x[3, 5] = float("inf")
    x[7, 10:] = torch.finfo(torch.float32).min
    s = -torch.rand(12, generator=torch.Generator().manual_seed(1)).cuda()
    s[5] = -float("inf")
    s[6] = float("nan")
    check(x, s, 4, 8)
    check(x, s, 2, 32)
    check(x, s, 12, 32)
    check(x[:4].contiguous(), torch.full((4,), -float("inf"), device="cuda"), 4, 9)       # nothing is alive


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_the_lowest_value(dtype):
    # a row of nothing but the type's lowest value is a uniform one; slices of it next to ordinary ones weigh nothing
    x = logits_of(4, 20000, dtype, 8)
    x[0] = torch.finfo(dtype).min
    x[1, :17000] = torch.finfo(dtype).min
    check(x, torch.zeros(4, device="cuda"), 2, 12)


@pytest.mark.parametrize("eos", [0, 2, 2999])
def test_finished_beams(eos):
    x = logits_of(8, 3000, torch.bfloat16, 9)
    s = -torch.rand(8, generator=torch.Generator().manual_seed(1)).cuda() * 5
    fin = torch.tensor([1, 0, 0, 1, 1, 1, 1, 1], dtype=torch.bool, device="cuda")
    s[7] = -float("inf")
    check(x, s, 4, 8, fin, eos)
    check(x, s, 4, 3, fin, eos)
    check(x, s, 2, 20, fin, eos)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,extra", [(1, 0), (0, 1), (3, 5), (8, 8)])
def test_rows_that_are_not_aligned(dtype, shift, extra):
    wide = logits_of(6, 10007 + shift + extra, dtype, 3)
    check(wide[:, shift:shift + 10007], torch.zeros(6, device="cuda"), 3, 6)


def test_same_bits_in_a_graph_and_beside_another_call():
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect, record_graph
    x, y, s = logits_of(16, 30000, torch.bfloat16, 1), logits_of(16, 30000, torch.bfloat16, 2), torch.zeros(16, device="cuda")
    a, b = SpindleKVBeamSelect(4, 4, 30000), SpindleKVBeamSelect(4, 4, 30000)
    want = [t.clone() for t in a.run(x, s)]
    other = [t.clone() for t in b.run(y, s)]
    graph = record_graph(lambda: a.run(x, s))
    for t in (a.score, a.parent, a.token):
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph.replay()
    b.run(y, s, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((a.score, a.parent, a.token), want))
    assert all(torch.equal(p, q) for p, q in zip((b.score, b.parent, b.token), other))


def test_scores_go_on_in_place():
    # the loop of a beam search: the scores of a step are the next step's, in the same buffer
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect
    select, plain = SpindleKVBeamSelect(6, 8, 20000), SpindleKVBeamSelect(6, 8, 20000)
    select.score.zero_()
    score = torch.zeros(48, device="cuda")
    for step in range(8):
        x = logits_of(48, 20000, torch.float32, step)
        select.run(x, select.score.view(-1))
        want = plain.run(x, score)
        assert all(torch.equal(p, q) for p, q in zip((select.score, select.parent, select.token), want))
        score = want[0].view(-1).clone()


def test_workspace_needs_no_preparation_and_serves_other_shapes():
    from paper_2507_06517_b200 import binding as B
    shapes = ((4, 8, 40000, 16), (1, 2, 300, 3), (2, 16, 9000, 32), (4, 8, 40000, 16))
    ws = torch.empty(max(B.spindlekv_beam_workspace_bytes(*s) for s in shapes), dtype=torch.uint8, device="cuda")
    for n, w, v, k in shapes:
        ws.random_(0, 256)
        x, s = logits_of(n * w, v, torch.float32, n + v), torch.zeros(n * w, device="cuda")
        out = torch.empty((n, k), device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda")
        for _ in range(3):
            B.spindlekv_beam_select(n, w, v, k, x, s, None, 0, *out, ws)
        want = R.beam(x.double().cpu().numpy(), np.zeros(n * w), w, k)
        assert np.array_equal(out[1].cpu().numpy(), want[1]) and np.array_equal(out[2].cpu().numpy(), want[2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_rows_whose_later_tiles_hold_the_best(dtype):
    # many blocks walk several tiles: rising logits (every tile exceeds the bound of the one before), a late plateau, a masked front
    n = 75
    x = torch.zeros((n, 100000), device="cuda")
    x[0::3] = torch.linspace(-4, 4, 100000, device="cuda")
    x[1::3, 60000:] = 3.0
    x[2::3, :90001] = -float("inf")
    x[2::3, 90001:] = logits_of(n // 3, 9999, torch.float32, 3)
    x += torch.arange(n, device="cuda")[:, None] % 3 * 0.25
    check(x.to(dtype), torch.zeros(n, device="cuda"), 3, 32)
    check(x.to(dtype)[:72], torch.zeros(72, device="cuda"), 8, 5)


def test_refusals():
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect
    with pytest.raises(ValueError):
        SpindleKVBeamSelect(1, 65, 100)
    with pytest.raises(ValueError):
        SpindleKVBeamSelect(1, 2, 3, 7)
    sel = SpindleKVBeamSelect(1, 2, 100)
    x, s = torch.zeros((2, 100), device="cuda"), torch.zeros(2, device="cuda")
    for bad in (x[:1], x.t().contiguous().t(), x.cpu(), torch.zeros((2, 101), device="cuda")):
        with pytest.raises(ValueError):
            sel.run(bad, s)
    with pytest.raises(ValueError):
        sel.run(x, s.double())
    with pytest.raises(ValueError):
        sel.run(x, s, finished=torch.zeros(2, device="cuda"))
    with pytest.raises(TypeError):
        sel.run(x.half(), s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,w,vocab,k", [(200, 4, 9001, 5), (1, 2, 400000, 32), (3000, 1, 40, 7)])
def test_more_rows_than_blocks_and_long_rows(dtype, n, w, vocab, k):
    check(logits_of(n * w, vocab, dtype, vocab), torch.zeros(n * w, device="cuda"), w, k)
