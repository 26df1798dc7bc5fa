"""Logits with penalties, biases and masks on the GPU against a form in 64 bits, one token at a time."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def reference(x, history=None, lens=None, n_prompt=None, repetition=None, presence=None, frequency=None, bias_token=None, bias_value=None, allowed=None):
    """float64 values, and how far an fp32 form of at most ``steps`` roundings may be off them."""
    x = x.double().cpu().numpy()
    n, v = x.shape
    z, off = x.copy(), np.zeros_like(x)
    get = lambda t, i, otherwise: otherwise if t is None else t[i].item()  # noqa: E731
    for i in range(n):
        if history is not None:
            h = history[i, : min(max(int(get(lens, i, history.shape[1])), 0), history.shape[1])].cpu().numpy()
            p = int(get(n_prompt, i, 0))
            inside = lambda a: a[(a >= 0) & (a < v)]  # noqa: E731
            seen = np.bincount(inside(h), minlength=v) > 0
            cnt = np.bincount(inside(h[max(p, 0):]), minlength=v)
            rep = get(repetition, i, 1.0)
            z[i] = np.where(seen, np.where(z[i] > 0, z[i] / rep, z[i] * rep), z[i])
            pen = get(frequency, i, 0.0) * cnt + get(presence, i, 0.0)
            off[i] = np.where(seen, np.abs(z[i]), 0) + np.where(cnt > 0, 2 * np.abs(pen) + np.abs(z[i]), 0)      # each rounding: half a step of 2^-23
            z[i] = np.where(cnt > 0, z[i] - pen, z[i])
        if bias_token is not None:
            for t, b in zip(bias_token[i].tolist(), bias_value[i].tolist()):
                if 0 <= t < v:
                    z[i, t] += b
                    off[i, t] += abs(z[i, t]) + abs(b)
        if allowed is not None:
            w = allowed[i if allowed.shape[0] > 1 else 0].cpu().numpy().view(np.uint32)
            t = np.arange(v)
            z[i] = np.where(w[t // 32] >> (t % 32).astype(np.uint32) & 1, z[i], -np.inf)
    return z, off * 2.0 ** -23


def check(x, out=None, **kw):
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    was = x.clone()
    want, off = reference(x, **{("lens" if k == "history_lens" else k): t for k, t in kw.items()})
    got = SpindleKVLogits(*x.shape).adjust(x, out=torch.empty_like(x) if out is None else out, **kw)
    torch.cuda.synchronize()
    if got.data_ptr() != x.data_ptr():
        assert torch.equal(torch.nan_to_num(x.float(), nan=5e9), torch.nan_to_num(was.float(), nan=5e9))
    g = got.double().cpu().numpy()
    fin = np.isfinite(want)
    assert np.array_equal(g[~fin], want[~fin], equal_nan=True)
    half = torch.finfo(x.dtype).eps / 2
    assert (np.abs(g - want)[fin] <= half * np.abs(want[fin]) + off[fin] * (1 + half) + 1e-38).all()
    return got


def logits(n, v, dtype, seed, stride=None, at=0):
    wide = torch.randn((n, (stride or v) + at), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda() * 3
    return wide[:, at:at + v]


def rules(n, v, hist, n_bias, seed, mask=True, far=False):
    gen = torch.Generator().manual_seed(seed)
    r = {}
    if hist:
        r["history"] = (torch.rand((n, hist), generator=gen) ** 3 * v).int()
        if far:
            r["history"][:, ::3] = torch.randint(-5, 2 * v, r["history"][:, ::3].shape, generator=gen, dtype=torch.int32)
        r["history_lens"] = torch.randint(0, hist + 1, (n,), generator=gen, dtype=torch.int32)
        r["n_prompt"] = torch.randint(0, hist + 1, (n,), generator=gen, dtype=torch.int32)
        r["repetition"] = torch.rand(n, generator=gen) + 0.7
        r["presence"], r["frequency"] = torch.randn(n, generator=gen), torch.rand(n, generator=gen)
    if n_bias:
        r["bias_token"] = torch.randint(-2, v + 2, (n, n_bias), generator=gen, dtype=torch.int32)
        r["bias_value"] = torch.randn((n, n_bias), generator=gen) * 4
    if mask:
        r["allowed"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, (v + 31) // 32), generator=gen, dtype=torch.int64).int()
    return {k: t.cuda() for k, t in r.items()}


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,v,hist,n_bias", [(1, 1, 1, 1), (3, 5, 0, 0), (2, 31, 7, 2), (5, 33, 100, 3), (1, 1000, 50, 0), (4, 32000, 300, 9), (7, 50257, 2000, 64),
                                             (130, 777, 40, 5), (2, 128256, 20000, 300), (3, 2049, 0, 5), (1, 300001, 1, 1)])
def test_all_rules_together(n, v, hist, n_bias, dtype):
    check(logits(n, v, dtype, v), **rules(n, v, hist, n_bias, v + 1))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("stride,at,out_stride,out_at", [(1001, 0, 1001, 0), (1003, 1, 1003, 1), (1000, 0, 1003, 3), (1007, 5, 1000, 0), (1008, 7, 1016, 3)])
def test_rows_of_any_stride_and_alignment(stride, at, out_stride, out_at, dtype):
    x, out = logits(4, 1000, dtype, 1, stride, at), logits(4, 1000, dtype, 2, out_stride, out_at)
    behind = out._base.clone()
    got = check(x, out=out, **rules(4, 1000, 200, 4, 3, far=True))
    behind[:, out_at:out_at + 1000] = got
    assert torch.equal(behind.view(torch.uint8), out._base.view(torch.uint8))               # nothing beside the rows


@pytest.mark.parametrize("dtype", [F32, BF])
def test_in_place_and_each_rule_alone(dtype):
    x = logits(5, 3001, dtype, 5)
    r = rules(5, 3001, 500, 6, 6)
    first = check(x.clone(), **r)
    assert torch.equal(check(x.clone(), out=None, **r).view(torch.uint8), first.view(torch.uint8))
    y = x.clone()
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    assert SpindleKVLogits(5, 3001).adjust(y, **r) is y and torch.equal(y.view(torch.uint8), first.view(torch.uint8))
    for names in (["allowed"], ["bias_token", "bias_value"], ["history", "repetition"], ["history", "presence", "history_lens"], ["history", "frequency", "n_prompt"], ["history"], []):
        check(x, **{k: r[k] for k in names})
    check(x, allowed=r["allowed"][:1].contiguous())
    check(x, allowed=r["allowed"].view(torch.uint32))
    check(x, history=r["history"][:, :0], repetition=r["repetition"])
    check(x, history=torch.cat([r["history"], r["history"]], 1)[:, 100:350], frequency=r["frequency"])
    check(x, history=r["history"], history_lens=torch.tensor([-4, 0, 10 ** 9, 1, 500], dtype=torch.int32).cuda(), n_prompt=torch.tensor([-1, 5, 10 ** 9, 0, 499], dtype=torch.int32).cuda(),
          presence=r["presence"])


@pytest.mark.parametrize("dtype", [F32, BF])
def test_masked_places_may_hold_anything_and_nothing_may_be_left(dtype):
    x = logits(4, 500, dtype, 8)
    r = rules(4, 500, 60, 3, 9)
    bits = (r["allowed"].long()[:, :, None] >> torch.arange(32, device="cuda") & 1).view(4, -1)[:, :500].bool()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min], device="cuda", dtype=dtype)[torch.arange(500, device="cuda") % 4]
    assert torch.equal(check(torch.where(bits, x, bad), **r), check(x, **r))
    r["allowed"] = torch.zeros_like(r["allowed"])
    assert (check(x, **r) == -float("inf")).all()
    # what is allowed keeps its infinities
    y = x.clone()
    y[:, 3], y[:, 4] = float("inf"), -float("inf")
    del r["allowed"]
    check(y, **r)


def test_the_same_tokens_many_times_over():
    x = logits(2, 4096, F32, 11)
    h = torch.full((2, 60000), 17, dtype=torch.int32, device="cuda")
    h[1, ::2] = 4095
    check(x, history=h, frequency=torch.tensor([0.01, 0.02], device="cuda"), presence=torch.tensor([1.0, -1.0], device="cuda"),
          bias_token=torch.full((2, 40), 17, dtype=torch.int32, device="cuda"), bias_value=torch.linspace(-1, 2, 80, device="cuda").view(2, 40))


def test_refusals_of_the_class():
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    with pytest.raises(ValueError):
        SpindleKVLogits(0, 10)
    a, x = SpindleKVLogits(3, 100), torch.zeros((3, 100), device="cuda")
    for kw in (dict(logits=x[:2]), dict(logits=x.t()), dict(logits=x.cpu()), dict(out=x.bfloat16()), dict(history=torch.zeros((3, 4), device="cuda")), dict(repetition=x[:, 0].contiguous()),
               dict(bias_token=torch.zeros((3, 2), dtype=torch.int32, device="cuda")), dict(allowed=torch.zeros((3, 3), dtype=torch.int32, device="cuda")),
               dict(history=torch.zeros((3, 4), dtype=torch.int32, device="cuda"), history_lens=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            a.adjust(**{"logits": x, **kw})


def test_offsets_beyond_32_bits():
    gap = 1717986918                                       # two rows are beyond 2^31 elements
    room = torch.empty(2 * gap + 5000, dtype=BF, device="cuda")
    x = torch.as_strided(room, (3, 5000), (gap, 1))
    x.copy_(logits(3, 5000, BF, 21))
    r = rules(3, 5000, 300, 5, 22)
    first = check(x.contiguous(), **r)
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    SpindleKVLogits(3, 5000).adjust(x, **r)
    assert torch.equal(x, first)
