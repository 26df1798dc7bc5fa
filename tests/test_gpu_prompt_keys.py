"""Prompt attention, key by key: that each one counts once, for the rows that see it, wherever parts, steps and tiles begin and end; batches of unlike layouts;
what is hidden, where keys are cut into parts."""
import math

import pytest
import torch

import prompt_ref as R
from paper_2507_06517_b200 import binding as B
from test_gpu_prompt import BF, F32, TYPES, attend, batch, check, make, tensor_of

pytestmark = pytest.mark.gpu

# lengths, rows (None: all), query heads, KV heads, d.  Few (row, query head) columns of a KV head go by themselves, the others by tiles; keys of calls with few rows are cut into parts
LONG = [
    ([5000], [1], 8, 8, 128), ([9001, 17, 4096], [1, 1, 1], 16, 8, 64), ([3000, 2049], [5, 3], 16, 8, 128), ([40000], [2], 8, 8, 128), ([777], [16], 8, 8, 64),
    ([5000], [40], 8, 8, 128), ([4097, 333], [33, 64], 16, 8, 64), ([40000], [19], 16, 8, 128), ([2500, 1000], [300, 300], 8, 8, 128), ([1300, 257], None, 16, 8, 128)]


def reach(lens, rows, packed):
    """``[(sequence, keys, rows, first row, keys that each row sees)]``."""
    out, r0 = [], 0
    for s, (n, r) in enumerate(zip(lens, rows or lens)):
        out.append((s, n, r, r0 if packed else 0, (n - r + 1 + torch.arange(r, device="cuda")).clamp(min=0)))
        r0 += r
    return out


def of(t, packed, s, first, n):
    """Rows of a sequence in the only layer: [heads, n, d]."""
    return t[0, first:first + n].transpose(0, 1) if packed else t[0, s, :, :n]


def lse_of(lse, rows, packed, s, first, n):
    at = first if packed else s * rows.max_len
    return lse[0, :, at:at + n].double()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("lens,rows,hq,h,d", LONG)
def test_every_key_counts_once(lens, rows, hq, h, d, packed, dtype):
    # Scores are zero, so a key's weight is one part in as many as the row sees; each key has an element of its own of a head's values, a thousand keys a call.  Sums of
    # ones are exact in every order; left are the reciprocal, the product and the result's rounding: half a step and 2^-22.  One key more or less is 2^-15.3 of 40000
    keys, rws, q, k, v = make(lens, rows, hq, h, d, dtype, packed, seed=61)
    k.zero_()
    half, many = torch.finfo(dtype).eps / 2, h * d
    at = torch.arange(many, device="cuda")
    first_keys = [sum(lens[:s]) if packed else 0 for s in range(len(lens))]
    for base in range(0, max(lens), many):
        v.zero_()
        for s, n in enumerate(lens):
            x = at[base + at < n]
            of(v, packed, s, first_keys[s], n)[x // d, base + x, x % d] = 1.0
        out, lse = attend(keys, rws, q, k, v)
        for s, n, r, r0, sees in reach(lens, rows, packed):
            seen = (base + at)[:, None] < sees                                     # [key of this call, row]
            want = torch.where(seen, 1.0 / sees.clamp(min=1).double(), 0.0).view(h, d, r).transpose(1, 2).repeat_interleave(hq // h, 0)
            got = of(out, packed, s, r0, r).double()
            assert ((got - want).abs() <= want * (half + 2.0 ** -21)).all()
            assert ((lse_of(lse, rws, packed, s, r0, r) - sees.double().log()).abs() <= 2.0 ** -21 * sees.double().log().clamp(min=1)).all()


def bits_of(t, d, dtype):
    """A row for each key that no other has: +1 and -1 by the bits of its number."""
    c = torch.arange(d, device="cuda") % 17
    return ((t[:, None] >> c & 1) * 2 - 1).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("lens,rows,hq,h,d", LONG)
def test_a_score_goes_with_its_own_key_and_value(lens, rows, hq, h, d, packed, dtype):
    # one key of a head outweighs all others by e^40: rows that see it give its value, the others the mean of what they see
    keys, rws, q, k, v = make(lens, rows, hq, h, d, dtype, packed, seed=62)
    q.fill_(1.0)
    half = torch.finfo(dtype).eps / 2
    hot_key = torch.tensor(40.0 / math.sqrt(d), dtype=dtype)
    score = hot_key.double().item() * math.sqrt(d)
    off = score * (d / 16 * (1 if dtype == BF else 6) + 4) * 2.0 ** -23             # the score's own roundings
    gen = torch.Generator().manual_seed(sum(lens))
    first_keys = [sum(lens[:s]) if packed else 0 for s in range(len(lens))]
    for s, n in enumerate(lens):
        of(v, packed, s, first_keys[s], n)[...] = bits_of(torch.arange(n, device="cuda"), d, dtype)
    most = max(lens)
    hot = [x for e in (0, 8, 16, 64, 128, 256, 512, 1024, 2048, 4096, most // 2, most - 1) for x in (e - 1, e, e + 1)] + torch.randint(0, most, (28,), generator=gen).tolist()
    for i in range(0, len(hot), h):
        mine = torch.tensor((hot[i:i + h] + hot)[:h], device="cuda").clamp(0, most - 1)
        k.zero_()
        for s, n in enumerate(lens):
            of(k, packed, s, first_keys[s], n)[torch.arange(h, device="cuda"), mine % n] = hot_key.to("cuda")
        out, lse = attend(keys, rws, q, k, v)
        for s, n, r, r0, sees in reach(lens, rows, packed):
            t = (mine % n).repeat_interleave(hq // h)                              # [query head]
            has = t[:, None] < sees
            bits = bits_of(torch.arange(n, device="cuda"), d, torch.float64)
            mean = (bits.cumsum(0)[(sees - 1).clamp(min=0)] / sees.clamp(min=1)[:, None]) * (sees > 0)[:, None]
            want = torch.where(has[:, :, None], bits[t][:, None], mean[None])
            got, lg = of(out, packed, s, r0, r).double(), lse_of(lse, rws, packed, s, r0, r)
            # its weight may stand above the reference, where bf16 rounds it; means are sums of ones
            assert ((got - want).abs() <= torch.where(has[:, :, None], (2 * half if dtype == BF else 0.0) + half + 2.0 ** -19, half * mean.abs() + 2.0 ** -20)).all()
            want_lse = torch.where(has, score + torch.log1p((sees - 1).clamp(min=0) * math.exp(-score)), sees.double().log())
            assert ((lg - want_lse).abs() <= torch.where(has, off + 2.0 ** -18, 2.0 ** -21 * want_lse.clamp(min=1))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows,hq,h,d", [([40000], [2], 8, 2, 128), ([5000], [1], 8, 8, 64), ([9000, 33], [5, 5], 4, 2, 128), ([4097], [33], 8, 2, 128), ([40000], [19], 4, 2, 64),
                                              ([2000, 900], None, 8, 2, 128)])
def test_sums_of_weights_to_the_scores_rounding(lens, rows, hq, h, d, dtype):
    # lse has no weights in bf16: a score's roundings (as in prompt_ref, 2^-23 of each of d / 16 sums and four steps behind them) and those of the sum
    keys, rws, q, k, v = make(lens, rows, hq, h, d, dtype, True, seed=63)
    lse = attend(keys, rws, q, k, v)[1]
    want = R.attend(q, k, v, keys, rws)[1]
    for (_, s, r0, r), (_, _, k0, n) in zip(R.spans(rws), R.spans(keys)):
        for head in range(hq):
            big = (q[0, r0:r0 + r, head].double().abs() @ k[0, k0:k0 + n, head // (hq // h)].double().abs().T / math.sqrt(d)).amax(-1)
            bound = big * (d / 16 * (1 if dtype == BF else 6) + 4) * 2.0 ** -23 + (n / 128 + 24) * 2.0 ** -23 + 2.0 ** -23 * want[0, head, r0:r0 + r].abs()
            assert ((lse[0, head, r0:r0 + r].double() - want[0, head, r0:r0 + r]).abs() <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows", [([700, 1, 0, 130, 2500], [2, 1, 2, 2, 2]), ([700, 1, 0, 130, 900], None), ([6000, 100, 3], [70, 40, 5]), ([600, 600], [600, 600])])
@pytest.mark.parametrize("packed_keys", [True, False])
def test_keys_and_rows_laid_out_unlike_one_another(lens, rows, packed_keys, dtype):
    gen = torch.Generator(device="cuda").manual_seed(64)
    for room_keys, room_rows, layers in ((0, 0, 1), (30, 0, 2), (0, 17, 1)):
        keys, rws = batch(lens, packed_keys, layers, room_keys), batch(rows or lens, not packed_keys, layers, room_rows)
        check(keys, rws, tensor_of(rws, 8, 128, dtype, gen), tensor_of(keys, 2, 128, dtype, gen), tensor_of(keys, 2, 128, dtype, gen))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows", [([6000], [40]), ([6000, 2500], [300, 70]), ([3000, 90], [130, 90])])
@pytest.mark.parametrize("packed", [True, False])
def test_hidden_values_where_keys_are_cut_into_parts(lens, rows, packed, dtype):
    hq, h, d = 4, 2, 128
    keys, rws, q, k, v = make(lens, rows, hq, h, d, dtype, packed, room=60, seed=65)
    taken_apart = 6 * d * (rws.total_len * hq + 2 * keys.total_len * h) if dtype == F32 else 0
    assert B.spindlekv_prompt_workspace_bytes(keys, rws, hq, h, d, B.BF16 if dtype == BF else B.F32) >= 256 + taken_apart + 2 * rws.total_len * hq * (d * 4 + 8)
    want, want_lse, bound = R.attend(q, k, v, keys, rws)
    for s, n in enumerate(lens):
        k0 = sum(lens[:s]) if packed else 0
        if not packed:
            k[0, s, :, n:], v[0, s, :, n:] = math.nan, math.inf
        vs = of(v, packed, s, k0, n)
        vs[0, n - 1], vs[1, n - 3, 5], vs[1, n - 2, 9] = math.nan, math.inf, -math.inf
    if packed:
        k[:, sum(lens):], v[:, sum(lens):] = math.inf, math.nan
    out, lse = attend(keys, rws, q, k, v)
    for s, n, r, r0, sees in reach(lens, rows, packed):
        got, exact, e = (of(t, packed, s, r0, r).double() for t in (out, want, bound))
        bad = torch.zeros_like(got, dtype=torch.bool)
        bad[:2, sees > n - 1] = True
        bad[2:, sees > n - 3, 5] = True
        bad[2:, sees > n - 2, 9] = True
        assert torch.equal(~got.isfinite(), bad)
        assert ((got - exact).abs()[~bad] <= e[~bad]).all()
        lg, lw = lse_of(lse, rws, packed, s, r0, r), lse_of(want_lse, rws, packed, s, r0, r)
        assert ((lg - lw).abs() <= 1e-4 * (1 + lw.abs())).all()
