"""Attention of prompts on the GPU against float64."""
import math

import pytest
import torch

import prompt_ref as R
from paper_2507_06517_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TYPES = [BF, F32]


def batch(lens, packed, n_layers=1, room=0):
    """A batch of these lengths: packed, padded, or (all alike) of equal lengths."""
    if packed:
        cu = torch.tensor([0] + lens).cumsum(0).int().cuda()
        return B.Batch(n_layers, len(lens), max(max(lens), 1), max(sum(lens) + room, max(lens), 1), cu)
    most = max(max(lens), 1) + room
    ll = None if min(lens) == most else torch.tensor([lens] * n_layers, dtype=torch.int32).cuda()
    return B.Batch(n_layers, len(lens), most, len(lens) * most, None, ll)


def tensor_of(b, heads, d, dtype, gen, size=1.0):
    shape = (b.n_layers, b.total_len, heads, d) if b.cu_seqlens is not None else (b.n_layers, b.n_seqs, heads, b.max_len, d)
    return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)


def make(lens, rows, hq, h, d, dtype, packed=False, n_layers=1, room=0, seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    keys, rws = batch(lens, packed, n_layers, room), batch(rows or lens, packed, n_layers, room)
    return keys, rws, tensor_of(rws, hq, d, dtype, gen, size), tensor_of(keys, h, d, dtype, gen), tensor_of(keys, h, d, dtype, gen)


def attend(keys, rows, q, k, v, scale=0.0, fill=7.0):
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    a = SpindleKVPromptAttention(keys, q.shape[2], k.shape[2], q.shape[-1], q.dtype, rows=rows)
    a.ws.fill_(0xA5)                                       # needs no preparation
    out = torch.full_like(q, fill)
    lse = torch.full((rows.n_layers, q.shape[2], rows.total_len), fill, device="cuda")
    a.run(q, k, v, out=out, lse=lse, scale=scale)
    assert a.status() == B.OK
    return out, lse


def check(keys, rows, q, k, v, scale=0.0):
    out, lse = attend(keys, rows, q, k, v, scale)
    want, want_lse, bound = R.attend(q, k, v, keys, rows, scale)
    there = ~want_lse.isnan()
    row = ~want.isnan()
    assert (out[~row] == 7.0).all() and (lse[~there] == 7.0).all()                          # nothing behind the last rows
    off = (out.double() - want).abs()[row]
    assert out[row].isfinite().all()
    assert (off <= bound[row]).all(), (off / bound[row].clamp(min=1e-300)).max()
    empty = want_lse == -math.inf
    assert (lse[empty] == -math.inf).all()
    ok = there & ~empty
    assert ((lse.double() - want_lse).abs()[ok] <= 1e-4 * (1 + want_lse.abs()[ok])).all()
    return out, lse


SHAPES = [  # lengths, rows (None: all), query heads, KV heads, d
    ([1], None, 1, 1, 64), ([1], None, 4, 2, 128), ([2], None, 8, 1, 128), ([127], None, 2, 2, 64), ([128], None, 2, 2, 128), ([129], None, 4, 4, 128),
    ([190], None, 4, 2, 64), ([257], None, 3, 1, 128), ([300], None, 7, 1, 128), ([515], None, 10, 2, 64), ([700], None, 16, 2, 128), ([1000], None, 5, 5, 128),
    ([2049], None, 8, 8, 128), ([333], None, 64, 1, 128), ([90], None, 128, 1, 64), ([150], None, 100, 1, 128),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows,hq,h,d", SHAPES)
def test_one_prompt(lens, rows, hq, h, d, dtype):
    check(*make(lens, rows, hq, h, d, dtype, seed=lens[0]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("packed,room", [(True, 0), (False, 0), (True, 37), (False, 50)])
@pytest.mark.parametrize("hq,h,d,layers", [(8, 2, 128, 1), (6, 2, 64, 2)])
def test_batches_of_uneven_prompts(packed, room, hq, h, d, layers, dtype):
    check(*make([130, 1, 0, 700, 64, 255, 0, 33], None, hq, h, d, dtype, packed, layers, room, seed=3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows", [([5000], [1]), ([3000, 17, 1], [1, 1, 1]), ([4097, 100], [33, 5]), ([2000], [300]), ([900, 64, 3], [20, 64, 0]), ([40000], [2])])
@pytest.mark.parametrize("packed", [True, False])
def test_last_rows_of_long_prompts(lens, rows, packed, dtype):
    check(*make(lens, rows, 8, 2, 128, dtype, packed, seed=5))


@pytest.mark.parametrize("lens,rows,hq,h,d", [
    ([4000], [1], 1, 1, 64), ([4000], [1], 7, 1, 128), ([2500, 3, 0, 9000], [5, 5, 5, 5], 8, 2, 64), ([2500, 3, 0, 9000], [5, 2, 0, 1], 4, 2, 128),
    ([7], [24], 2, 2, 128), ([5000], [24], 1, 1, 128), ([5000], [25], 1, 1, 128), ([6, 8, 9, 31], [3, 3, 3, 3], 8, 1, 64)])
@pytest.mark.parametrize("packed", [True, False])
def test_few_columns_of_a_head(lens, rows, hq, h, d, packed):
    # fp32 with few rows and query heads: one pass over the keys, up to 24 columns
    keys, rws, q, k, v = make(lens, rows, hq, h, d, F32, packed, 2, seed=41)
    check(keys, rws, q, k, v)
    if packed and min(lens) > 0:                           # the rows of a head behind one another
        move = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)
        check(keys, rws, q, move(k), move(v))


@pytest.mark.parametrize("lens,rows,hq,h,d", [
    ([4000], [1], 1, 1, 64), ([4000], [1], 7, 1, 128), ([2500, 3, 0, 9000], [5, 5, 5, 5], 8, 2, 64), ([2500, 3, 0, 9000], [5, 2, 0, 1], 4, 2, 128),
    ([7], [24], 2, 2, 128), ([5000], [3], 5, 1, 128), ([5000], [16], 1, 1, 64), ([5000], [17], 2, 2, 128), ([6, 8, 9, 31], [3, 3, 3, 3], 8, 1, 64), ([15, 16, 17, 33], [1, 1, 1, 1], 8, 2, 128)])
@pytest.mark.parametrize("packed", [True, False])
def test_few_columns_of_a_head_in_bf16(lens, rows, hq, h, d, packed):
    keys, rws, q, k, v = make(lens, rows, hq, h, d, BF, packed, 2, seed=43)
    check(keys, rws, q, k, v)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,hq", [(3000, 5, 2), (1000, 8, 1), (37, 3, 4), (16, 2, 6)])
def test_values_that_some_of_few_columns_do_not_see(n, rows, hq, dtype):
    # the last row alone sees the last value: the others' results are those without it
    keys, rws, q, k, v = make([n, n], [rows, rows], hq, 1, 128, dtype, True, seed=44)
    want, want_lse = attend(keys, rws, q, k, v)
    for odd in (math.nan, math.inf):
        w = v.clone()
        w[0, n - 1], w[0, 2 * n - 1] = odd, odd
        out, lse = attend(keys, rws, q, k, w)
        last = torch.zeros(2 * rows, dtype=torch.bool, device="cuda")
        last[rows - 1], last[2 * rows - 1] = True, True
        assert not out[:, last].isfinite().any()
        bound = R.attend(q, k, v, keys, rws)[2]
        assert ((out.double() - want.double()).abs()[:, ~last] <= 2 * bound[:, ~last]).all()
        assert torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 40])
def test_a_nan_that_is_seen_shows_whatever_its_weight(rows, dtype):
    # keys cut into parts; one key outweighs all others by 2^400
    keys, rws, q, k, v = make([6000], [rows], 8, 2, 128, dtype, False, seed=45)
    q[...], k[...] = 1.0, 0.0
    k[..., 100, :] = 25.0
    v[0, 0, 1, 5000, 7] = math.nan
    out, lse = attend(keys, rws, q, k, v)
    assert out[..., 7][0, 0, 4:].isnan().all() and out[0, 0, :4].isfinite().all() and out[..., :7].isfinite().all()
    assert ((out[0, 0, :4].double() - v[0, 0, 0, 100].double()).abs() <= 2 ** -7 * v[0, 0, 0, 100].double().abs()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows,packed", [([300, 70, 1, 0, 129], None, False), ([300, 70, 1, 0, 129], None, True), ([3000, 1700], [40, 33], False), ([2000, 100], [2, 2], False)])
def test_scratch_full_of_nans(lens, rows, packed, dtype):
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    keys, rws, q, k, v = make(lens, rows, 8, 2, 128, dtype, packed, room=0 if rows else 50, seed=46)
    a = SpindleKVPromptAttention(keys, 8, 2, 128, dtype, rows=rws)
    a.ws.fill_(0xFF)
    out = torch.full_like(q, 7.0)
    a.run(q, k, v, out=out)
    want, _, bound = R.attend(q, k, v, keys, rws)
    row = ~want.isnan()
    assert a.status() == B.OK and (out[~row] == 7.0).all()
    assert ((out.double() - want).abs()[row] <= bound[row]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_see_nothing(dtype):
    # more rows than keys: the first ones see none
    check(*make([3, 0, 500], [10, 4, 700], 4, 2, 64, dtype, False, seed=6))
    check(*make([0], [5], 4, 2, 128, dtype, False, seed=6))
    check(*make([2], [300], 4, 1, 128, dtype, True, seed=6))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_sequences(dtype):
    gen = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 40, (300,), generator=gen).tolist()
    check(*make(lens, None, 4, 2, 64, dtype, True, seed=8))
    check(*make(lens[:150], None, 4, 2, 128, dtype, False, 2, seed=8))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("packed,layers", [(True, 1), (False, 2)])
def test_many_sequences_of_several_blocks(packed, layers, dtype):
    # more sequences than a warp has lanes, whose blocks are found from one item to the next
    gen = torch.Generator().manual_seed(2)
    lens = torch.randint(0, 500, (70,), generator=gen).tolist()
    check(*make(lens, None, 16, 2, 64, dtype, packed, layers, seed=21))


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_every_size(dtype):
    # references that move late, and by much; scores all alike; a scale of one's own
    keys, rows, q, k, v = make([900], None, 4, 2, 128, dtype, seed=9, size=6.0)
    ramp = torch.linspace(0.1, 4.0, 900, device="cuda")[:, None]
    check(keys, rows, q, (k * ramp).to(dtype), v)
    check(keys, rows, q, (k * ramp.flip(0)).to(dtype), v, scale=0.3)
    check(keys, rows, torch.zeros_like(q), k, v)
    check(keys, rows, q, k, v, scale=1e-6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows,packed", [([300, 200], None, False), ([300, 200], None, True), ([3000], [5], False)])
def test_what_a_row_does_not_see_may_be_anything(lens, rows, packed, dtype):
    keys, rws, q, k, v = make(lens, rows, 4, 2, 128, dtype, packed, room=60, seed=11)
    check(keys, rws, q, k, v)
    want, _, bound = R.attend(q, k, v, keys, rws)
    # behind the sequences
    for t in (k, v):
        if packed:
            t[:, sum(lens):] = math.nan
            t[:, sum(lens) + 20:] = math.inf
        else:
            for s, n in enumerate(lens):
                t[:, s, :, n:] = math.inf if s else math.nan
    check(keys, rws, q, k, v)
    # the last key: only the last row sees it
    last = (0, sum(lens) - 1) if packed else (0, len(lens) - 1, slice(None), lens[-1] - 1)
    k[last], v[last] = math.nan, math.inf
    out, lse = attend(keys, rws, q, k, v)
    n_r = (rows or lens)[-1]
    got, want, bound = (x[0, -60 - n_r:-60] if packed else x[0, -1].transpose(0, 1)[:n_r] for x in (out, want, bound))
    assert got[-1].isnan().all()
    assert got[:-1].isfinite().all()
    assert ((got.double() - want).abs()[:-1] <= bound[:-1]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_numbers_show_where_they_are_seen(dtype):
    keys, rows, q, k, v = make([1000], None, 2, 1, 64, dtype, seed=12)
    # what does not see them is the formula's, to the formula's bound: tiles that are done by hand add d / 8 + 3 products to a score and 128 to a
    # result one after the other, 19 and 128 steps of 2^-24 where the bound counts 28 and 375 (bf16: 8 and 62, and half a step of 2^-8 beside them)
    want, bound = (x[0, 0] for x in R.attend(q, k, v, keys, rows)[::2])
    v[0, 0, 0, 400, 7] = math.nan
    v[0, 0, 0, 700, 9] = -math.inf
    out, lse = attend(keys, rows, q, k, v)
    assert lse.isfinite().all()
    bad = ~out[0, 0].isfinite()                                # [heads, rows, d]
    seen = torch.zeros_like(bad)
    seen[:, 400:, 7] = True
    seen[:, 700:, 9] = True
    assert torch.equal(bad, seen)
    assert ((out[0, 0].double() - want).abs()[~bad] <= bound[~bad]).all()
    v.fill_(math.nan)                                          # and all of them
    assert attend(keys, rows, q, k, v)[0].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_streams_graphs_and_repeats(dtype):
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention, record_graph
    gen = torch.Generator(device="cuda").manual_seed(13)
    n, hq, h, d = 450, 8, 2, 128
    keys = batch([n, n], False)
    wide = torch.randn((1, 2, n, hq + 2 * h, d), generator=gen, device="cuda").to(dtype)    # a fused projection's rows: [token][q, k, v heads]
    q, k, v = (wide[:, :, :, a:b].transpose(2, 3) for a, b in ((0, hq), (hq, hq + h), (hq + h, hq + 2 * h)))
    first = check(keys, keys, q, k, v)
    assert all(torch.equal(a, b) for a, b in zip(first, attend(keys, keys, q.contiguous(), k.contiguous(), v.contiguous())))
    out = torch.full((1, 2, n, hq, d), 7.0, dtype=dtype, device="cuda").transpose(2, 3)
    a = SpindleKVPromptAttention(keys, hq, h, d, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.run(q, k, v, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, first[0])
    graph = record_graph(lambda: a.run(q, k, v, out=out))
    wide.copy_(wide.flip(2))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, attend(keys, keys, q, k, v)[0])
    assert a.status() == B.OK


@pytest.fixture
def limits():
    yield B.spindlekv_set_tuning
    for key in (B.TUNE_MBAR_WAIT_CYCLES, B.TUNE_PAGED_WITHHOLD):
        B.spindlekv_set_tuning(key, -1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,rows,blocks", [([300, 200, 90], None, (0, 3, 5)), ([3000], [3], (0, 7))])
def test_a_wait_that_gives_up_shows_in_the_status_and_leaves_nothing_behind(lens, rows, blocks, dtype, limits):
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention, record_graph
    keys, rws, q, k, v = make(lens, rows, 4, 2, 128, dtype, True, seed=21)
    a = SpindleKVPromptAttention(keys, 4, 2, 128, dtype, rows=rws)
    want, _, bound = R.attend(q, k, v, keys, rws)
    out = torch.zeros_like(q)
    for block in blocks:                                   # whichever block gives up, and whatever the scratch held
        a.ws.random_(0, 256)
        limits(B.TUNE_MBAR_WAIT_CYCLES, 2_000_000)
        limits(B.TUNE_PAGED_WITHHOLD, block)
        a.run(q, k, v, out=out)
        assert a.status() == B.TIMEOUT
        limits(B.TUNE_MBAR_WAIT_CYCLES, -1)
        limits(B.TUNE_PAGED_WITHHOLD, -1)
        for _ in range(2):
            a.run(q, k, v, out=out)
            assert a.status() == B.OK
            assert ((out.double() - want).abs() <= bound).all()
    graph = record_graph(lambda: a.run(q, k, v, out=out))
    for _ in range(3):
        a.ws.random_(0, 256)
        graph.replay()
        graph.replay()
        assert a.status() == B.OK


@pytest.mark.parametrize("dtype", TYPES)
def test_offsets_beyond_32_bits(dtype):
    # layers 1.2 * 2^31 elements apart
    keys, rows, q, k, v = make([200, 90], None, 4, 2, 64, dtype, False, n_layers=2, seed=31)
    far, gap = [], 2576980480
    room = torch.empty(gap + 3 * q[0].numel(), dtype=dtype, device="cuda")
    at = 0
    for t in (q, k, v):
        f = torch.as_strided(room, t.shape, (gap, *t.stride()[1:]), at)
        f.copy_(t)
        far.append(f)
        at += t[0].numel()
    first = check(keys, rows, q, k, v)
    assert all(torch.equal(a, b) for a, b in zip(first, attend(keys, rows, *far)))


def test_objects_side_by_side_on_two_streams():
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    sets = [make([700, 300], None, 8, 2, 128, dt, True, seed=s) for s, dt in ((41, BF), (42, F32))] + [make([3000], [4], 8, 2, 128, BF, False, seed=43)]
    want = [attend(*s)[0] for s in sets]
    objects = [SpindleKVPromptAttention(s[0], 8, 2, 128, s[2].dtype, rows=s[1]) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [torch.full_like(s[2], 7.0) for s in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for a, s, st, o in zip(objects, sets, streams, outs):
            a.run(*s[2:], out=o, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want)) and all(a.status() == B.OK for a in objects)


def test_refusals_of_the_class_and_what_it_makes_itself():
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
    keys, rows, q, k, v = make([40, 17], None, 4, 2, 64, BF, False, seed=51)
    with pytest.raises(TypeError):
        SpindleKVPromptAttention(keys, 4, 2, 64, torch.float16)
    with pytest.raises(ValueError):
        SpindleKVPromptAttention(keys, 4, 3, 64, BF)
    with pytest.raises(ValueError):
        SpindleKVPromptAttention(B.Batch(1, 2, 40, 80, None, keys.layer_lens.cpu()), 4, 2, 64, BF)
    a = SpindleKVPromptAttention(keys, 4, 2, 64, BF)
    for kw in (dict(q=q.float()), dict(q=q[:, :, :3]), dict(K=k[:, :, :, :39]), dict(V=v.cpu()), dict(K=k.transpose(3, 4).contiguous().transpose(3, 4)),
               dict(out=q[:, :1]), dict(lse=torch.zeros((1, 4, 79), device="cuda")), dict(lse=torch.zeros((1, 4, 80), device="cuda", dtype=BF))):
        with pytest.raises(ValueError):
            a.run(**{"q": q, "K": k, "V": v, **kw})
    with pytest.raises(B.SpindleKVError):
        a.run(q, k, v, out=q)
    with pytest.raises(B.SpindleKVError):
        a.run(q, k, v, scale=-1.0)
    out = a.run(q, k, v)
    assert (out[0, 1, :, 17:] == 0).all() and torch.equal(out[0, 1, :, :17], attend(keys, rows, q, k, v)[0][0, 1, :, :17])


@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows_far_apart(dtype):
    # the second layer 1.2 * 2^31 elements behind the first
    keys, rows, q, k, v = make([700, 90], [3, 3], 4, 2, 64, dtype, False, n_layers=2, seed=32)
    far, gap = [], 2576980480
    room = torch.empty(gap + q[0].numel() + k[0].numel() + v[0].numel(), dtype=dtype, device="cuda")
    at = 0
    for t in (q, k, v):
        f = torch.as_strided(room, t.shape, (gap, *t.stride()[1:]), at)
        f.copy_(t)
        far.append(f)
        at += t[0].numel()
    first = check(keys, rows, q, k, v)
    assert all(torch.equal(a, b) for a, b in zip(first, attend(keys, rows, *far)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_rows", [2, 70])
def test_a_recorded_call_follows_the_lengths_on_the_device(n_rows, dtype):
    from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention, record_graph
    gen = torch.Generator(device="cuda").manual_seed(47)
    lens = torch.tensor([[2000, 5, 900]], dtype=torch.int32, device="cuda")
    keys, rows = B.Batch(1, 3, 2500, 7500, None, lens), B.Batch(1, 3, n_rows, 3 * n_rows, None, torch.full_like(lens, n_rows))
    q, k, v = tensor_of(rows, 8, 128, dtype, gen), tensor_of(keys, 2, 128, dtype, gen), tensor_of(keys, 2, 128, dtype, gen)
    a = SpindleKVPromptAttention(keys, 8, 2, 128, dtype, rows=rows)
    out = torch.full_like(q, 7.0)
    graph = record_graph(lambda: a.run(q, k, v, out=out))
    for now, new in (([2000, 5, 900], [n_rows] * 3), ([2500, 0, 1], [n_rows, 0, 1]), ([130, 2499, 64], [1, n_rows, n_rows])):
        lens.copy_(torch.tensor([now]))
        rows.layer_lens.copy_(torch.tensor([new]))
        out.fill_(7.0)
        graph.replay()
        assert a.status() == B.OK
        want, _, bound = R.attend(q, k, v, keys, rows)
        row = ~want.isnan()
        assert (out[~row] == 7.0).all() and ((out.double() - want).abs()[row] <= bound[row]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_more_sequences_than_a_grid_of_few_rows_takes(dtype):
    # 9000 sequences x 8 heads go by whole tiles, the first hundred of them by themselves
    gen = torch.Generator(device="cuda").manual_seed(48)
    lens = torch.randint(0, 21, (1, 9000), generator=gen, dtype=torch.int32, device="cuda")
    keys, rows = B.Batch(1, 9000, 20, 180000, None, lens), B.Batch(1, 9000, 1, 9000)
    q, k, v = tensor_of(rows, 8, 64, dtype, gen), tensor_of(keys, 8, 64, dtype, gen), tensor_of(keys, 8, 64, dtype, gen)
    out, lse = attend(keys, rows, q, k, v)
    some = B.Batch(1, 100, 20, 2000, None, lens[:, :100].contiguous()), B.Batch(1, 100, 1, 100)
    want, want_lse, bound = R.attend(q[:, :100], k[:, :100], v[:, :100], *some)
    assert ((out[:, :100].double() - want).abs() <= bound).all()
    check(*some, q[:, :100].contiguous(), k[:, :100].contiguous(), v[:, :100].contiguous())
    assert out.isfinite().all() and (out[0, (lens == 0)[0]] == 0).all() and ((lse == -math.inf) == (lens == 0)[0]).all()
