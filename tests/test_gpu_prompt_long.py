"""Prompt attention over very long keys, bf16: sums do not shrink with the number of keys."""
import math

import pytest
import torch

import prompt_ref as R
from paper_2507_06517_b200 import binding as B
from test_gpu_prompt import BF, attend, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,rows,hq,h,d", [(131072, 600, 32, 8, 128), (140001, 1200, 16, 4, 64), (131072, 570, 32, 8, 128), (300000, 130, 8, 2, 128)])
def test_sums_keep_their_size(n, rows, hq, h, d):
    # Values of one sign, of another size in each element, so that results lie anywhere between two numbers of bf16.  Their mean deviation beside that of the rounded formula: 16384 keys
    # are 1024 products of 16 keys added to a sum that may be cut off by 2^-22 of it each time, 2^-12; more keys than that have to be summed up without
    gen = torch.Generator(device="cuda").manual_seed(n)
    q = torch.randn((1, 1, hq, rows, d), generator=gen, device="cuda").to(BF)
    k = (torch.randn((1, 1, h, n, d), generator=gen, device="cuda") * 0.3).to(BF)
    size = 2.0 ** (torch.rand((1, 1, h, 1, d), generator=gen, device="cuda") * 4)
    v = ((torch.randn((1, 1, h, n, d), generator=gen, device="cuda") * 0.3 + 1.0) * size).to(BF)
    out, _ = attend(B.Batch(1, 1, n, n), B.Batch(1, 1, rows, rows), q, k, v)
    off = count = 0.0
    for head in range(0, hq, hq // h):
        for r0 in range(0, rows, 128):
            x = q[0, 0, head, r0:r0 + 128].double() @ k[0, 0, head * h // hq].double().T / math.sqrt(d)
            x += torch.full_like(x, -math.inf).triu(n - rows + r0 + 1)
            want = torch.softmax(x, -1) @ v[0, 0, head * h // hq].double()
            off += ((out[0, 0, head, r0:r0 + 128].double() - want.to(BF).double()) / want).sum().item()
            count += want.numel()
    assert abs(off / count) <= 2.0 ** -12, off / count


@pytest.mark.parametrize("lens,rows,hq,h,d,packed", [
    ([40000], [300], 8, 2, 128, False), ([16384, 16385, 33000], [700, 700, 700], 32, 4, 64, True), ([50001, 100, 16513], [129, 100, 2000], 16, 4, 128, False),
    ([16512], [16512], 4, 1, 128, False)])
def test_long_keys_to_the_formula(lens, rows, hq, h, d, packed):
    check(*make(lens, rows, hq, h, d, BF, packed, seed=71))


def test_references_that_move_far_apart():
    # scores that rise, fall and rise again by far more than a reference may lag; what was summed earlier is weighed anew
    n, rows = 70000, 1100
    keys, rws, q, k, v = make([n], [rows], 16, 2, 128, BF, False, seed=72)
    ramp = torch.cat([torch.linspace(0, 3, 30000, device="cuda"), torch.linspace(3, 0.1, 20000, device="cuda"), torch.linspace(0.1, 6, 20000, device="cuda")])
    for r in (ramp, ramp.flip(0)):
        check(keys, rws, q, (k * r[:, None]).to(BF), v)
    # keys that no score gives any weight for the first 20000
    low = k.clone()
    low[:, :, :, :20000] = -math.inf
    q = q.abs()
    out, lse = attend(keys, rws, q, low, v)
    want, want_lse, bound = R.attend(q, k[:, :, :, 20000:].contiguous(), v[:, :, :, 20000:].contiguous(), B.Batch(1, 1, n - 20000, n - 20000), rws)
    assert ((out.double() - want).abs() <= bound).all() and ((lse.double() - want_lse).abs() <= 1e-4 * (1 + want_lse.abs())).all()


@pytest.mark.parametrize("n,hidden_from", [(40000, 39930), (40000, 39999), (32808, 32807), (32808, 32760)])
def test_hidden_values_behind_long_keys(n, hidden_from):
    # (32808: the tiles that hide keys lie on both sides of where 256 of them are summed)
    rows = 900
    keys, rws, q, k, v = make([n], [rows], 32, 4, 128, BF, False, seed=73)
    want, _, bound = R.attend(q, k, v, keys, rws)
    v[0, 0, :, hidden_from, 3], v[0, 0, :, n - 1, 4] = math.nan, math.inf
    out, _ = attend(keys, rws, q, k, v)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[..., hidden_from - n + rows:, 3] = True
    bad[..., rows - 1, 4] = True
    assert torch.equal(~out.isfinite(), bad)
    assert ((out.double() - want).abs()[~bad] <= bound[~bad]).all()


def test_scratch_full_of_nans_and_one_object_for_long_and_short():
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    lens = torch.tensor([[40000, 200]], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(74)
    q, k, v = (torch.randn((1, 2, x, m, 64), generator=gen, device="cuda").to(BF) for x, m in ((16, 1200), (4, 40000), (4, 40000)))
    keys, rows = B.Batch(1, 2, 40000, 80000, None, lens), B.Batch(1, 2, 1200, 2400, None, lens.clamp(max=1200))
    a = SpindleKVPromptAttention(keys, 16, 4, 64, BF, rows=rows)
    a.ws.fill_(0xFF)
    for now in ([40000, 200], [200, 39999], [16385, 16384]):
        lens.copy_(torch.tensor([now]))
        rows.layer_lens.copy_(lens.clamp(max=1200))
        out = torch.full_like(q, 7.0)
        a.run(q, k, v, out=out)
        assert a.status() == B.OK
        want, _, bound = R.attend(q, k, v, keys, rows)
        row = ~want.isnan()
        assert (out[~row] == 7.0).all() and ((out.double() - want).abs()[row] <= bound[row]).all()


def test_a_wait_that_gives_up_over_long_keys():
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    keys, rws, q, k, v = make([40000], [900], 32, 4, 128, BF, False, seed=75)
    a = SpindleKVPromptAttention(keys, 32, 4, 128, BF, rows=rws)
    want, _, bound = R.attend(q, k, v, keys, rws)
    out = torch.zeros_like(q)
    for block in (0, 77):
        a.ws.random_(0, 256)
        try:
            B.spindlekv_set_tuning(B.TUNE_MBAR_WAIT_CYCLES, 2_000_000)
            B.spindlekv_set_tuning(B.TUNE_PAGED_WITHHOLD, block)
            a.run(q, k, v, out=out)
            assert a.status() == B.TIMEOUT
        finally:
            for key in (B.TUNE_MBAR_WAIT_CYCLES, B.TUNE_PAGED_WITHHOLD):
                B.spindlekv_set_tuning(key, -1)
        a.run(q, k, v, out=out)
        assert a.status() == B.OK and ((out.double() - want).abs() <= bound).all()
