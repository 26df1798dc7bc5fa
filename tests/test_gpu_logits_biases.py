"""Long lists of biases: bit for bit the fp32 operations in the stated order, in time that grows with the list and not with its square."""
import numpy as np
import pytest
import torch

from test_gpu_logits import BF, F32, logits, rules

pytestmark = pytest.mark.gpu


def in_order(x, r):
    """The rules in fp32, each operation rounded by itself, biases one after the other; then x's type."""
    z = x.float().cpu().numpy().copy()
    n, v = z.shape
    f = np.float32
    for i in range(n):
        if "history" in r:
            h = r["history"][i, : int(r["history_lens"][i])].cpu().numpy()
            p = int(r["n_prompt"][i])
            inside = lambda a: a[(a >= 0) & (a < v)]  # noqa: E731
            seen, cnt = (np.bincount(inside(a), minlength=v) for a in (h, h[p:]))
            rep, pres, freq = (f(r[k][i].item()) for k in ("repetition", "presence", "frequency"))
            z[i] = np.where(seen > 0, np.where(z[i] > 0, z[i] / rep, z[i] * rep), z[i])
            z[i] = np.where(cnt > 0, z[i] - (freq * cnt.astype(f) + pres), z[i])
        with np.errstate(invalid="ignore"):
            for t, b in zip(r["bias_token"][i].tolist(), r["bias_value"][i].cpu().numpy()):
                if 0 <= t < v:
                    z[i, t] = z[i, t] + b
        if "allowed" in r:
            t = np.arange(v)
            z[i] = np.where(r["allowed"][i].cpu().numpy().view(np.uint32)[t // 32] >> (t % 32).astype(np.uint32) & 1, z[i], f(-np.inf))
    return torch.from_numpy(z).to(x.dtype)


def same(got, want):
    return torch.equal(torch.nan_to_num(got.float().cpu(), nan=5e9), torch.nan_to_num(want.float(), nan=5e9))


def adjusted(x, r, **kw):
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    return SpindleKVLogits(*x.shape).adjust(x, **kw, **r)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,v,hist,n_bias,mask", [
    (3, 2500, 50, 64, True), (3, 2500, 50, 65, True), (2, 1000, 50, 512, True), (2, 1000, 50, 513, True), (3, 5000, 300, 5000, False), (2, 7, 5, 2000, False), (1, 1, 1, 700, False), (2, 40000, 0, 1025, False),
    (1, 128256, 20000, 3001, True), (4, 20001, 100, 1537, True)])
def test_biases_are_added_in_the_order_of_the_list(n, v, hist, n_bias, mask, dtype):
    x, r = logits(n, v, dtype, v), rules(n, v, hist, n_bias, v + n_bias, mask)
    # several to a token, of sizes at which another order gives another sum; tokens outside the vocabulary among them
    gen = torch.Generator(device="cuda").manual_seed(n_bias)
    r["bias_value"] *= torch.pow(10.0, torch.randint(-3, 5, r["bias_value"].shape, generator=gen, device="cuda"))
    r["bias_token"][:, ::3] = (r["bias_token"][:, ::3].clamp(0, v - 1) % 11) * max(v // 11, 1) % v
    r["bias_token"][0, ::50], r["bias_token"][0, 1::50] = -1, v
    want = in_order(x, r)
    assert same(adjusted(x, r, out=torch.full_like(x, 7.0)), want)
    y = x.clone()
    assert same(adjusted(y, r), want) and same(y, want)                           # in place


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("stride,at,out_stride,out_at", [(5001, 0, 5001, 0), (5003, 1, 5003, 1), (5007, 5, 5000, 0)])
def test_long_lists_over_rows_of_any_alignment(stride, at, out_stride, out_at, dtype):
    x, out = logits(3, 5000, dtype, 1, stride, at), logits(3, 5000, dtype, 2, out_stride, out_at)
    r = rules(3, 5000, 200, 900, 3)
    r["bias_token"][:, 100:400] = r["bias_token"][:, 400:700]
    assert same(adjusted(x, r, out=out), in_order(x, r))


@pytest.mark.parametrize("n_bias", [8, 1300])
def test_biases_that_cancel_and_biases_that_are_no_numbers(n_bias):
    x = logits(2, 1200, F32, 4)
    r = {"bias_token": torch.arange(n_bias, device="cuda", dtype=torch.int32).remainder(1200).repeat(2, 1)}
    r["bias_value"] = -x.gather(1, r["bias_token"].long())                         # zeros are left
    r["bias_value"][0, 3], r["bias_value"][0, 4], r["bias_value"][1, 5] = -float("inf"), float("inf"), float("nan")
    got, want = adjusted(x, r, out=torch.full_like(x, 7.0)), in_order(x, r)
    assert same(got, want) and (got[:, min(n_bias, 1200) - 1] == 0).all()          # (a longer list begins again: its first tokens have two)


def test_time_grows_with_the_list_and_not_with_its_square():
    # a bias for every token: 2 x 131072.  As many comparisons as tokens times biases of a slice would be 3.4e10: 18 ms
    v = 131072
    x, out = logits(2, v, F32, 5), torch.empty((2, v), device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(6)
    r = {"bias_token": torch.stack([torch.randperm(v, generator=gen, device="cuda") for _ in range(2)]).int(), "bias_value": torch.randn((2, v), generator=gen, device="cuda")}
    from paper_2507_06517_b200.pipeline import SpindleKVLogits
    a, times = SpindleKVLogits(2, v), []
    for _ in range(4):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        a.adjust(x, out=out, **r)
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    assert torch.equal(out, x.scatter_add(1, r["bias_token"].long(), r["bias_value"]))
    assert min(times) < 8.0, times
