"""The 8-bit paged cache on the GPU against float64 forms: codes, scales, tables and reference counts exactly, attention within
bounds derived from its roundings."""
import numpy as np
import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().double().cpu().numpy()


def make(n_layers, n_seqs, hq, h, d, n_pages, max_pages, ps, fmt, seed=0):
    """A cache whose memory holds leftovers: every byte pattern in the codes, NaN in the scales."""
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache
    c = SpindleKVPagedCache(n_layers, n_seqs, hq, h, d, n_pages, max_pages, ps, fmt)
    gen = torch.Generator().manual_seed(seed)
    k, v, ks, vs, _ = c.pool.tensors
    for t in (k, v):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=gen, dtype=torch.int32).to(torch.uint8))
    for t in (ks, vs):
        t.fill_(float("nan"))
    c.pages.fill_(2 ** 31 - 1)
    return c


def ref_of(c):
    k, v, ks, vs, ref = (t.view(torch.uint8) if i < 2 else t for i, t in enumerate(c.pool.tensors))
    return R.RefCache(*(x.cpu().numpy() for x in (k, v, ks, vs, ref, c.pages, c.lens)), "int8" if c.pool.c.format == 0 else "e4m3")


def same_state(c, r):
    now = ref_of(c)
    for what in ("ref", "lens", "pages"):
        assert np.array_equal(getattr(now, what), getattr(r, what)), what
    for g in "kv":
        assert np.array_equal(now.scale[g].view(np.uint32) & 0x7FFFFFFF, r.scale[g].view(np.uint32) & 0x7FFFFFFF) \
            or np.array_equal(now.scale[g], r.scale[g], equal_nan=True), g
        assert np.array_equal(now.codes[g], r.codes[g]), g


def lens_t(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows(shape, dtype, seed, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=gen) * torch.exp(spread * torch.randn(shape[:-1] + (1,), generator=gen))
    return x.to(DT[dtype]).cuda()


def fill(c, lens, dtype="bf16", seed=1, spread=1.0):
    """Gives the sequences these lengths and writes random rows into what is new; the reference does the same."""
    r = ref_of(c)
    start = r.resize(np.array(lens))
    assert start is not None
    c.resize(lens_t(lens))
    n = max(1, int((np.array(lens) - start).max()))
    K, V = (rows((c.n_layers, c.n_seqs, c.Hkv, n, c.d), dtype, seed + i, spread) for i in (0, 100))
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    return r


# ---- append ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,ps", [(64, 16), (128, 64)])
def test_append_writes_the_same_codes_and_scales(fmt, dtype, d, ps):
    c = make(2, 4, None, 3, d, 60, 240 // ps, ps, fmt)
    r = ref_of(c)
    was = r.lens.copy()
    # nothing, one token, a block's end and beyond it; then on from there, with larger values so that open blocks are rescaled
    for step, (lens, spread) in enumerate([([[0, 1, 15, 16], [17, 33, 47, 64]], 0.5), ([[1, 2, 16, 17], [17, 34, 90, 65]], 2.0),
                                           ([[1, 30, 50, 17], [80, 35, 100, 66]], 3.0), ([[2, 31, 51, 18], [81, 36, 101, 67]], 3.0)]):
        r = fill(c, lens, dtype, seed=10 * step, spread=spread)
        assert c.status() == 0
        same_state(c, r)
    assert not np.array_equal(was, r.lens)


def test_append_takes_rows_in_any_order_and_from_strided_tensors():
    fmt, d, h, n = "int8", 128, 2, 50
    c = make(2, 3, None, h, d, 40, 4, 32, fmt)
    lens = [[50, 7, 0], [33, 16, 50]]
    r = ref_of(c)
    start = r.resize(np.array(lens))
    c.resize(lens_t(lens))
    # token-major tensors [L, B, row, head, d] with a gap behind every row; rows picked from 70 by lists with numbers outside
    K, V = (rows((2, 3, 70, h, 2 * d), "bf16", s)[..., :d].transpose(2, 3) for s in (1, 2))
    idx = torch.randint(-3, 75, (2, h, 3 * n), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    c.append(K, V, idx=idx)
    r.append(start, f64(K), f64(V), idx.cpu().numpy(), n)
    same_state(c, r)
    c.append(K, V, start=lens_t([[-1, 7, 3], [40, -1, 50]]), max_new=50)      # nothing but tokens 40 .. 49 of none: start >= lens or < 0
    same_state(c, r)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_append_shows_a_nan_or_infinity_in_the_blocks_scale(fmt, bad):
    c = make(1, 2, None, 1, 64, 8, 2, 32, fmt)
    fill(c, [[20, 20]], "f32")
    r = ref_of(c)
    start = r.resize(np.array([[21, 38]]))
    c.resize(lens_t([[21, 38]]))
    K, V = rows((1, 2, 1, 18, 64), "f32", 5), rows((1, 2, 1, 18, 64), "f32", 6)
    K[0, 0, 0, 0, 63] = bad
    V[0, 1, 0, 17, 0] = bad
    c.append(K, V)
    r.append(start, np.where(np.isfinite(f64(K)), f64(K), np.nan), np.where(np.isfinite(f64(V)), f64(V), np.nan))
    same_state(c, r)
    assert np.isnan(r.scale["k"]).sum() > 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_of_zeros_and_of_the_smallest_and_largest_numbers(fmt):
    c = make(1, 5, None, 1, 64, 8, 1, 32, fmt)
    r = ref_of(c)
    start = r.resize(np.full((1, 5), 16))
    c.resize(lens_t([[16] * 5]))
    K = torch.randn((1, 5, 1, 16, 64), generator=torch.Generator().manual_seed(1)).cuda()
    for s, f in enumerate((0.0, 1e-44, 1e-38, 1e-30, 1e37)):
        K[0, s] *= f
    K[0, 4, 0, 0, 0] = 3.4e38
    c.append(K, -K)
    r.append(start, f64(K), f64(-K))
    same_state(c, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_int8_codes_on_exact_halves_go_to_even(dtype):
    # amax 127 gives scale 1: k + 1/2 must go to the even neighbour, whatever the reciprocal rounds to
    c = make(1, 1, None, 1, 128, 4, 1, 16, "int8")
    r = ref_of(c)
    start = r.resize(np.array([[16]]))
    c.resize(lens_t([[16]]))
    K = (torch.arange(16 * 128) % 254 / 2 - 63.5).view(1, 1, 1, 16, 128).to(DT[dtype]).cuda()
    K[..., 0, 0] = 127
    V = K * 3                                       # scale 3: quotients that only nearly are halves
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    same_state(c, r)


def test_append_leaves_out_tokens_on_pages_outside_the_pool():
    c = make(1, 2, None, 1, 64, 8, 4, 16, "int8")
    r = fill(c, [[40, 40]])
    c.pages[0, 0, 1] = -7
    c.pages[0, 1, 2] = 8
    before = ref_of(c)
    K = rows((1, 2, 1, 40, 64), "bf16", 9)
    c.append(K, K, start=lens_t([[0, 0]]))
    after = ref_of(c)
    for s, gone in ((0, 1), (1, 2)):
        assert np.array_equal(after.codes["k"][r.pages[0, s, gone]], before.codes["k"][r.pages[0, s, gone]])
        assert not np.array_equal(after.codes["k"][r.pages[0, s, 0]], before.codes["k"][r.pages[0, s, 0]])


# ---- attention ---------------------------------------------------------------------------------------------------

def check_attention(c, r, q, out, dtype, scale=None):
    """|error| <= half a step of the output type, plus A = sum of weight * |value| times: the weight's rounding to fp16 pieces (2^-12
    for one, 2^-22 for two), and twice the relative error of a weight.  That is the absolute error of its score: d + 16 fp32
    additions and products, each 2^-23 of S = sum |q_i k_i| * scale at most (the tensor cores cut off where a sum would round), the query's own pieces
    (2^-22 of S, fp32 only) and 2^-20 for the power function and the score's own fp32 step (scores below 16 here).  What fades out of
    fp16 is below 2^-30 of the largest value per token."""
    want, mag, top = r.attend(f64(q), scale)
    got = f64(out)
    half = torch.finfo(DT[dtype]).eps / 2
    weight = 2.0 ** -12 if dtype == "bf16" else 2.0 ** -22
    err = ((c.d + 16) * 2.0 ** -23 + (0 if dtype == "bf16" else 2.0 ** -22)) * top[..., None] + 2.0 ** -20
    big = max(np.nanmax(np.abs(r.rows("v", l, s)[0]), initial=0.0) for l, s in r.units())
    bound = half * np.abs(want) + mag * (weight + 2 * err) * 1.01 + r.lens.max() * big * 2.0 ** -30
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / np.maximum(bound, 1e-300)).max()
    assert worst <= 1, worst


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,ps,h,hn,n_rows", [(128, 64, 2, 4, 1), (64, 16, 3, 1, 1), (128, 32, 1, 8, 1), (64, 128, 2, 7, 2), (128, 16, 2, 8, 3),
                                             (128, 64, 1, 5, 5), (64, 32, 2, 8, 16), (128, 128, 1, 8, 16), (128, 16, 4, 2, 4)])
def test_attention_matches_float64(fmt, dtype, d, ps, h, hn, n_rows):
    c = make(2, 6, hn * h, h, d, 2 * 6 * (640 // ps), 640 // ps, ps, fmt)
    r = fill(c, [[0, 1, 15, 16, 17, 333], [2, 5, 31, 64, 130, 640]], dtype, spread=0.3)
    q = rows((2, 6, hn * h, n_rows, d), dtype, 77, 0.2)
    out = c.attend(q, max_len=640)
    check_attention(c, r, q, out, dtype)
    seen = r.lens[:, :, None] - n_rows + 1 + np.arange(n_rows)
    assert (f64(out).transpose(0, 1, 3, 2, 4)[seen <= 0] == 0).all()        # rows that see nothing


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_len", [1, 700, 100000])
def test_attention_over_many_runs_whatever_the_length_hint(dtype, max_len):
    # one unit over many runs, runs over several units, and a hint far from the truth
    c = make(1, 3, 8, 2, 128, 400, 320, 16, "int8")
    r = fill(c, [[5000, 3, 700]], dtype, spread=0.3)
    q = rows((1, 3, 8, 1, 128), dtype, 5, 0.2)
    check_attention(c, r, q, c.attend(q, max_len=max_len), dtype)


@pytest.mark.parametrize("max_len", [40, 250, 100000])
@pytest.mark.parametrize("n_layers,n_seqs", [(2, 16), (3, 41)])
def test_attention_of_many_short_sequences(n_layers, n_seqs, max_len):
    # more sequences than lanes, many of them empty; a block per unit, or runs with several units in each
    c = make(n_layers, n_seqs, 4, 2, 64, n_layers * n_seqs * 16, 16, 16, "e4m3")
    rng = np.random.default_rng(n_seqs)
    lens = np.where(rng.random((n_layers, n_seqs)) < 0.3, 0, rng.integers(1, 251, (n_layers, n_seqs)))
    r = fill(c, lens.tolist(), spread=0.3)
    q = rows((n_layers, n_seqs, 4, 2, 64), "bf16", 5, 0.2)
    out = torch.full_like(q, 7.0)
    c.attend(q, out=out, max_len=max_len)
    check_attention(c, r, q, out, "bf16")
    assert c.status() == 0


def test_one_workspace_serves_attention_of_every_shape():
    c = make(1, 2, None, 2, 128, 64, 16, 32, "int8")
    r = fill(c, [[500, 33]], spread=0.3)
    from paper_2507_06517_b200.binding import SpindleKVError
    with pytest.raises(SpindleKVError):
        c.attend(rows((1, 2, 4, 17, 128), "bf16", 1))
    c.ws_attend = None
    for hq, n_rows, dtype in ((16, 16, "f32"), (2, 1, "bf16"), (6, 5, "bf16"), (16, 1, "f32")):
        q = rows((1, 2, hq, n_rows, 128), dtype, 5, 0.2)
        if c.ws_attend is not None:
            c.ws_attend.random_(0, 256)                   # it needs no preparation
        check_attention(c, r, q, c.attend(q), dtype)


def test_attention_with_very_uneven_scales():
    # a value of 1e30 that has no weight must not drown the others, nor one of 1e-30 with all of it
    c = make(1, 2, 2, 1, 64, 20, 4, 32, "int8")
    K, V = torch.zeros((1, 2, 1, 100, 64), device="cuda"), rows((1, 2, 1, 100, 64), "f32", 3, 0.1)
    K[0, 0, 0, 40, 0] = -1e4
    V[0, 0, 0, 40] = 1e30
    K[0, 1, 0, 40, 0] = 1e4
    V[0, 1, 0, 40] = 1e-30
    r = ref_of(c)
    start = r.resize(np.full((1, 2), 100))
    c.resize(lens_t([[100, 100]]))
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = torch.zeros((1, 2, 2, 1, 64), device="cuda")
    q[..., 0] = 1.0
    got, (want, mag, _) = f64(c.attend(q)), r.attend(f64(q))
    assert (np.abs(got - want) <= 1e-5 * mag + 1e-45).all()
    # the value of 1e-30 shares a block, and so a scale, with values near 1: its code is 0
    assert np.abs(want[0, 0]).max() < 10 and (want[0, 1] == 0).all()


def test_attention_with_a_block_of_tiny_values():
    # all the weight on a block of its own scale, 1e-30 of its neighbours'
    c = make(1, 1, 2, 1, 64, 20, 4, 32, "e4m3")
    K, V = torch.zeros((1, 1, 1, 100, 64), device="cuda"), rows((1, 1, 1, 100, 64), "f32", 3, 0.1)
    K[0, 0, 0, 32:48, 0] = 1e4
    V[0, 0, 0, 32:48] *= 1e-30
    r = ref_of(c)
    start = r.resize(np.full((1, 1), 100))
    c.resize(lens_t([[100]]))
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = torch.zeros((1, 1, 2, 1, 64), device="cuda")
    q[..., 0] = 1.0
    got, (want, mag, _) = f64(c.attend(q)), r.attend(f64(q))
    assert (np.abs(got - want) <= 1e-5 * mag).all() and 0 < np.abs(want).max() < 1e-29


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_attention_with_tiny_and_huge_queries(dtype, size):
    c = make(1, 1, 4, 1, 128, 8, 2, 64, "e4m3")
    r = fill(c, [[90]], dtype, spread=0.3)
    q = (rows((1, 1, 4, 1, 128), "f32", 5, 0.2) * size).to(DT[dtype])
    check_attention(c, r, q, c.attend(q, scale=0.1 / size), dtype, scale=0.1 / size)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("of_q,of_k,of_v", [(122, -120, 0), (-118, 116, 0), (0, 0, 118), (0, 0, -116)])
def test_attention_of_numbers_near_the_ends_of_fp32(fmt, dtype, of_q, of_k, of_v):
    # the scores and the results are ordinary numbers (or at least fp32 ones): no product or sum on the way may leave fp32's range
    c = make(1, 1, 4, 1, 128, 8, 4, 64, fmt)
    r = ref_of(c)
    start = r.resize(np.array([[200]]))
    c.resize(lens_t([[200]]))
    K, V = rows((1, 1, 1, 200, 128), dtype, 1, 0.3) * 2.0 ** of_k, rows((1, 1, 1, 200, 128), dtype, 2, 0.3) * 2.0 ** of_v
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 1, 4, 1, 128), dtype, 5, 0.2) * 2.0 ** of_q
    check_attention(c, r, q, c.attend(q, scale=0.02), dtype, scale=0.02)


@pytest.mark.parametrize("fmt,ps", [("int8", 16), ("e4m3", 32), ("int8", 64), ("e4m3", 128)])
@pytest.mark.parametrize("h,hn,n_rows", [(2, 6, 3), (1, 8, 4), (2, 7, 6), (1, 8, 8), (1, 7, 10), (2, 8, 16)])
def test_attention_of_many_columns(fmt, ps, h, hn, n_rows):
    # 18 to 128 columns, lengths around a tile's end and over many tiles, more units than runs and the reverse, whatever the hint
    tiles = [[0, 1, 127, 128, 129, 511], [513, 5, 3000, 16, 640, 1100]]
    c = make(2, 6, hn * h, h, 128, 6400 // ps + 12, 3200 // ps, ps, fmt)
    r = fill(c, tiles, spread=0.3)
    q = rows((2, 6, hn * h, n_rows, 128), "bf16", 77, 0.2)
    first = None
    for max_len in (600, 3000, 100000):
        out = torch.full_like(q, 7.0)
        c.attend(q, out=out, max_len=max_len)
        check_attention(c, r, q, out, "bf16")
        assert c.status() == 0
        again = torch.full_like(q, 7.0)
        c.attend(q, out=again, max_len=max_len)
        assert torch.equal(out, again)
        first = out if first is None else first
    seen = r.lens[:, :, None] - n_rows + 1 + np.arange(n_rows)
    assert (f64(first).transpose(0, 1, 3, 2, 4)[seen <= 0] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("rising", [False, True])
def test_attention_of_many_columns_moves_its_references(fmt, rising):
    # scores and values whose sizes rise, or fall, from block to block: every tile moves the running maximum, and the unit of the sums
    c = make(1, 1, 8, 1, 128, 40, 36, 64, fmt)
    n = 2000
    r = ref_of(c)
    start = r.resize(np.array([[n]]))
    c.resize(lens_t([[n]]))
    K, V = rows((1, 1, 1, n, 128), "bf16", 1, 0.1), rows((1, 1, 1, n, 128), "bf16", 2, 0.1)
    size = torch.arange(n, device="cuda").div(64, rounding_mode="floor").float()
    size = size if rising else size.max() - size
    K = (K * 0.1 * size[:, None]).to(K.dtype)
    V = (V * torch.exp2(size / 4)[:, None]).to(V.dtype)
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 1, 8, 4, 128), "bf16", 5, 0.2)
    check_attention(c, r, q, c.attend(q), "bf16")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("of_q,of_k,of_v", [(122, -120, 0), (-118, 116, 0), (0, 0, 118), (0, 0, -116)])
def test_attention_of_many_columns_near_the_ends_of_fp32(fmt, of_q, of_k, of_v):
    c = make(1, 1, 8, 1, 128, 24, 12, 64, fmt)
    r = ref_of(c)
    start = r.resize(np.array([[700]]))
    c.resize(lens_t([[700]]))
    K, V = rows((1, 1, 1, 700, 128), "bf16", 1, 0.3) * 2.0 ** of_k, rows((1, 1, 1, 700, 128), "bf16", 2, 0.3) * 2.0 ** of_v
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 1, 8, 5, 128), "bf16", 5, 0.2) * 2.0 ** of_q
    check_attention(c, r, q, c.attend(q, scale=0.02), "bf16", scale=0.02)


def test_attention_of_many_columns_with_nan_infinities_and_missing_pages():
    c = make(1, 3, 16, 2, 128, 100, 40, 32, "e4m3")
    fill(c, [[900, 1001, 32]], "f32", spread=0.3)
    r = ref_of(c)
    start = r.resize(np.array([[901, 1002, 33]]))
    c.resize(lens_t([[901, 1002, 33]]))
    K, V = rows((1, 3, 2, 1, 128), "f32", 1), rows((1, 3, 2, 1, 128), "f32", 2)
    K[0, 2, 1] = float("nan")
    V[0, 0, 0] = float("inf")
    c.append(K, V)
    q = rows((1, 3, 16, 3, 128), "bf16", 3)
    q[0, 1, 3, 1, 7] = float("nan")
    q[0, 1, 9, 0, 100] = float("-inf")
    c.pages[0, 1, 5] = -1
    c.pages[0, 1, 6] = 100
    got = f64(c.attend(q))
    nan = np.isnan(got).all(-1)
    want = np.zeros((1, 3, 16, 3), bool)
    want[0, 2, 8:, 2] = want[0, 0, :8, 2] = True           # the last row alone sees a new token: blocks 56 and 2 begin with it
    want[0, 1, 3, 1] = want[0, 1, 9, 0] = True
    # sequence 0's new token is the 901st, in a block with four earlier ones: the rows that see these are lost as well
    want[0, 0, :8] = True
    assert np.array_equal(nan, want) and np.isfinite(got[~want]).all()
    r.append(start, np.nan_to_num(f64(K)), np.where(np.isinf(f64(V)), 0, f64(V)))
    r.pages[0, 1, 5:7] = -1
    clean, mag, _ = r.attend(np.nan_to_num(f64(q), neginf=0.0))
    # half a step of bf16, and less than that of the sum of weight * |value| for the weights
    assert (np.abs(got - clean)[~want] <= (2.0 ** -8 * np.abs(clean) + 2.0 ** -8 * mag)[~want]).all()


def test_attention_of_poisoned_blocks_reaches_only_rows_that_see_them():
    c = make(1, 2, 4, 2, 64, 16, 3, 16, "int8")
    fill(c, [[32, 32]], "f32", spread=0.3)
    r = ref_of(c)
    start = r.resize(np.full((1, 2), 33))
    c.resize(lens_t([[33, 33]]))
    K, V = rows((1, 2, 2, 1, 64), "f32", 1), rows((1, 2, 2, 1, 64), "f32", 2)
    K[0, 0, 1] = float("nan")
    V[0, 1, 0] = float("inf")
    c.append(K, V)
    q = rows((1, 2, 4, 2, 64), "f32", 3)
    got = f64(c.attend(q))
    nan = np.isnan(got).all(-1)
    want = np.zeros((1, 2, 4, 2), bool)
    want[0, 0, 2:, 1] = want[0, 1, :2, 1] = True           # the last row alone, of the KV head that holds it
    assert np.array_equal(nan, want)
    r.append(start, np.nan_to_num(f64(K)), np.where(np.isinf(f64(V)), 0, f64(V)))
    clean, _, _ = r.attend(f64(q))
    assert np.abs(got - clean)[~want].max() < 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_nan_or_infinite_queries_keeps_to_their_rows(dtype):
    c = make(1, 1, 4, 1, 64, 8, 4, 16, "int8")
    r = fill(c, [[50]], dtype, spread=0.3)
    q = rows((1, 1, 4, 2, 64), dtype, 3)
    clean = f64(c.attend(q).clone())
    q[0, 0, 1, 0, 5] = float("nan")
    q[0, 0, 2, 1, 7] = float("inf")
    got = f64(c.attend(q))
    bad = np.zeros((1, 1, 4, 2), bool)
    bad[0, 0, 1, 0] = bad[0, 0, 2, 1] = True
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], clean[~bad])
    assert r.lens[0, 0] == 50


def test_attention_leaves_out_tokens_on_pages_outside_the_pool():
    c = make(1, 2, 4, 2, 128, 16, 8, 16, "e4m3")
    fill(c, [[100, 20]], spread=0.3)
    c.pages[0, 0, 2] = -1
    c.pages[0, 0, 4] = 16
    c.pages[0, 1, :] = 1 << 30                     # none left: zeros
    q = rows((1, 2, 4, 1, 128), "bf16", 4, 0.2)
    out = c.attend(q)
    check_attention(c, ref_of(c), q, out, "bf16")
    assert (out[0, 1] == 0).all()


def test_attention_clamps_lengths_to_the_table():
    c = make(1, 2, 2, 1, 64, 8, 2, 16, "int8")
    r = fill(c, [[32, 32]], spread=0.3)
    c.lens.copy_(lens_t([[2 ** 31 - 1, -5]]))
    q = rows((1, 2, 2, 1, 64), "bf16", 4, 0.2)
    out = c.attend(q)
    r.lens = np.array([[32, 0]])
    check_attention(c, r, q, out, "bf16")


def test_attention_strides_streams_graphs_and_bits():
    from paper_2507_06517_b200.pipeline import record_graph
    c = make(2, 3, 8, 2, 128, 200, 64, 32, "int8")
    r = fill(c, [[1000, 40, 2000], [16, 999, 1]], spread=0.3)
    wide = rows((2, 3, 3, 8, 2 * 128), "bf16", 4, 0.2)
    q = wide[..., :128].transpose(2, 3)                           # [L, B, Hq, rows, d], token-major with a gap
    held = torch.full((2, 3, 3, 8, 2 * 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = held[..., 128:].transpose(2, 3)
    c.attend(q, out=out)
    check_attention(c, r, q, out, "bf16")
    assert (held[..., :128] == 7).all()
    first = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    c.attend(q, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    graph = record_graph(lambda: c.attend(q, out=out))
    out.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    for layer in range(2):                                        # one layer at a time, from the same table
        got = c.attend(q[layer:layer + 1].contiguous(), layer=layer, max_len=2000)
        r1 = ref_of(c)
        r1.pages, r1.lens, r1.n_layers = r1.pages[layer:layer + 1], r1.lens[layer:layer + 1], 1
        check_attention(c, r1, q[layer:layer + 1], got, "bf16")


def test_attention_over_a_pool_beyond_four_gigabytes():
    # the pages of one sequence at both ends of a pool whose byte offsets pass 32 bits
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache
    n = (5 << 30) // (8 * 128 * 128)
    c = SpindleKVPagedCache(1, 1, 8, 8, 128, n, 8, 128, "int8")
    c.pages.copy_(torch.tensor([[[n - 1, 0, n - 2, 1, n // 2, n - 3, 2, n - 4]]], dtype=torch.int32))
    c.page_ref[c.pages.view(-1).long()] = 1
    c.lens.fill_(1000)
    K, V = rows((1, 1, 8, 1000, 128), "bf16", 1, 0.3), rows((1, 1, 8, 1000, 128), "bf16", 2, 0.3)
    c.append(K, V, start=lens_t([[0]]))
    q = rows((1, 1, 8, 1, 128), "bf16", 4, 0.2)
    got = c.attend(q).clone()
    small = SpindleKVPagedCache(1, 1, 8, 8, 128, 8, 8, 128, "int8")
    small.resize(lens_t([[1000]]))
    small.append(K, V)
    assert torch.equal(got, small.attend(q))
    assert int(c.compact()) == 8
    assert torch.equal(c.attend(q), got)


def test_attention_of_many_columns_strides_streams_graphs_and_a_large_pool():
    # pages at both ends of a pool whose byte offsets pass 32 bits; token-major queries with gaps; another stream; two graphs of one
    # cache replayed in turn; one layer at a time
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache, record_graph
    n = (5 << 30) // (4 * 64 * 128)
    c = SpindleKVPagedCache(2, 2, 32, 4, 128, n, 20, 64, "e4m3")
    small = SpindleKVPagedCache(2, 2, 32, 4, 128, 80, 20, 64, "e4m3")
    lens = [[1200, 77], [640, 1281 - 1]]
    r = fill(small, lens, spread=0.3)
    far = torch.randperm(80, generator=torch.Generator().manual_seed(1)).cuda()
    far = torch.where(far % 2 == 0, far, n - 1 - far).int()        # page i of the small pool lies at far[i]
    for big, little in zip(c.pool.tensors, small.pool.tensors):
        big[far.long()] = little
    c.pages.copy_(torch.where(small.pages >= 0, far[small.pages.clamp(min=0).long()], small.pages))
    c.lens.copy_(small.lens)
    wide = rows((2, 2, 5, 32, 2 * 128), "bf16", 4, 0.2)
    q = wide[..., 128:].transpose(2, 3)                           # [L, B, Hq, rows, d]
    held = torch.full((2, 2, 5, 32, 2 * 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = held[..., :128].transpose(2, 3)
    c.attend(q, out=out)
    check_attention(c, r, q, out, "bf16")
    assert (held[..., 128:] == 7).all() and torch.equal(out, small.attend(q.contiguous()))
    first = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    c.attend(q, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    other = torch.zeros_like(first)
    graphs = [record_graph(lambda: c.attend(q, out=out)), record_graph(lambda: c.attend(q, out=other, max_len=700))]
    out.zero_()
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    check_attention(c, r, q, other, "bf16")
    for layer in range(2):
        got = c.attend(q[layer:layer + 1], layer=layer, max_len=2000)
        r1 = R.RefCache(r.codes["k"], r.codes["v"], r.scale["k"], r.scale["v"], r.ref, r.pages[layer:layer + 1], r.lens[layer:layer + 1], "e4m3")
        check_attention(c, r1, q[layer:layer + 1], got, "bf16")
    assert c.status() == 0


# ---- pages -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,ps,d,h", [("int8", 16, 64, 3), ("e4m3", 64, 128, 2)])
def test_random_histories_of_page_operators(fmt, ps, d, h):
    rng = np.random.default_rng(ps)
    c = make(3, 7, 2 * h, h, d, 150, 5, ps, fmt)
    for step in range(25):
        r = ref_of(c)
        what = rng.integers(0, 4)
        if what == 0:
            lens = rng.integers(0, 5 * ps + 1, (3, 7))
            fits = r.resize(lens)
            c.resize(lens_t(lens))
            if fits is None:
                assert c.status() == 4 and (c.start == -1).all()           # capacity
            else:
                assert c.status() == 0 and np.array_equal(c.start.cpu().numpy(), fits)
                n = max(1, int((lens - fits).max()))
                K, V = rows((3, 7, h, n, d), "bf16", step), rows((3, 7, h, n, d), "bf16", step + 50)
                c.append(K, V)
                r.append(fits, f64(K), f64(V))
        elif what == 1:
            add = int(rng.integers(-3, 4))
            ok = r.resize(r.lens + add)
            c.resize(add=add)
            assert c.status() == (0 if ok is not None else 1 if (r.lens + add < 0).any() or (r.lens + add > 5 * ps).any() else 4)
            if ok is not None:          # what a new token holds before it is written is nobody's business
                K, V = rows((3, 7, h, 3, d), "bf16", step), rows((3, 7, h, 3, d), "bf16", step + 50)
                c.append(K, V)
                r.append(ok, f64(K), f64(V))
        elif what == 2:
            parent = rng.integers(-1 if rng.random() < 0.3 else 0, 7, 7)
            ok = r.fork(parent)
            c.fork(lens_t(parent))
            assert c.status() == (0 if ok else 4)
        else:
            assert int(c.compact()) == r.compact()
            assert c.status() == 0
        same_state(c, r)
        n = int((r.ref > 0).sum())
        counted = np.zeros_like(r.ref)
        for l, s in r.units():
            np.add.at(counted, r.pages[l, s, :r.count(r.lens[l, s])], 1)
        assert np.array_equal(counted, r.ref) and n <= 150                 # every reference is a table entry


def test_page_operators_refuse_on_the_device_and_change_nothing():
    c = make(1, 3, 2, 1, 64, 4, 4, 16, "int8")
    r = fill(c, [[20, 16, 16]])
    for lens in ([[20, 16, 17]], [[20, 16, 65]], [[20, -1, 16]], [[2 ** 31 - 1, 0, 0]]):
        c.resize(lens_t(lens))
        assert c.status() == (4 if lens[0][2] == 17 else 1)
        assert (c.start == -1).all()
        c.append(rows((1, 3, 1, 8, 64), "bf16", 1), rows((1, 3, 1, 8, 64), "bf16", 1))      # start -1: nothing is written
        same_state(c, r)
    for parent, why in (([0, 0, 1], 4), ([0, 1, 3], 1), ([-2, 1, 2], 1)):
        c.fork(lens_t(parent))
        assert c.status() == why
        same_state(c, r)
    c.resize(c.no_tokens)
    assert c.status() == 0 and (c.page_ref == 0).all()


def test_fork_of_many_sequences_and_of_wide_tables():
    # more sequences than threads of a copying block, tables wider than a tile, full and open pages
    c = make(2, 300, 2, 1, 64, 9000, 75, 16, "int8")
    rng = np.random.default_rng(1)
    lens = np.where(rng.random((2, 300)) < 0.03, rng.integers(1, 75 * 16 + 1, (2, 300)), rng.integers(0, 40, (2, 300)))
    r = fill(c, lens.tolist())
    parent = rng.integers(-1, 300, 300)
    assert r.fork(parent)
    c.fork(lens_t(parent))
    assert c.status() == 0
    same_state(c, r)


def test_page_operators_in_a_graph():
    from paper_2507_06517_b200.pipeline import record_graph
    c = make(2, 4, 2, 1, 64, 64, 8, 16, "e4m3")
    fill(c, [[20, 3, 0, 17], [1, 1, 40, 2]])
    r = ref_of(c)
    parent = lens_t([1, 0, 2, 2])
    K, V = rows((2, 4, 1, 1, 64), "bf16", 1), rows((2, 4, 1, 1, 64), "bf16", 2)

    def step():
        c.fork(parent)
        c.resize(add=1)
        c.append(K, V)

    graph = record_graph(step)          # runs once beforehand
    graph.replay()
    torch.cuda.synchronize()
    for _ in range(2):
        assert r.fork([1, 0, 2, 2])
        start = r.resize(r.lens + 1)
        r.append(start, f64(K), f64(V))
    assert c.status() == 0
    same_state(c, r)


# ---- as they are used --------------------------------------------------------------------------------------------

def test_python_layer_refuses_before_launching():
    c = make(2, 3, 4, 2, 64, 16, 4, 16, "int8")
    q = rows((2, 3, 4, 1, 64), "bf16", 1)
    with pytest.raises(ValueError):
        c.attend(q.cpu())
    with pytest.raises(ValueError):
        c.attend(q[:1])
    with pytest.raises(ValueError):
        c.attend(q, out=q[:, :, :2])
    with pytest.raises(IndexError):
        c.attend(q[:1], layer=2)
    with pytest.raises(ValueError):
        c.fork(torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        c.resize(torch.zeros((2, 3), dtype=torch.int32))
    with pytest.raises(ValueError):
        c.append(q, q)
    with pytest.raises(ValueError):
        c.append(q[:, :, :2], q[:, :, :2], idx=torch.zeros((2, 3, 3), dtype=torch.int32, device="cuda"))
    from paper_2507_06517_b200.binding import SpindleKVError
    with pytest.raises(SpindleKVError):
        c.attend(rows((2, 3, 4, 17, 64), "bf16", 1))


def test_evicted_prompt_decodes_from_the_paged_cache():
    # eviction of a prompt, what it kept stored in 8 bits, then decoding with beams: fork, resize, append, attend per layer.
    # The float64 reference takes the same steps from the rows that eviction kept
    from gpu_util import generate, make_config, stack_layers, torch_dtype
    from paper_2507_06517_b200 import synth
    from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect, SpindleKVPagedCache, SpindleKVPass
    wl = synth.Workload("paged", 3, 1, 8, 2, 128, "bf16", 32, (700, 700), 40, (0.05, 0.3), 4, "recency", budget_tokens=200.0, seed=21)
    host = generate(wl)
    p = SpindleKVPass(make_config(wl), wl.seq_lens, torch_dtype(wl))
    layers = [0, 1, 2]
    K, V = stack_layers(wl, host, layers, "K"), stack_layers(wl, host, layers, "V")
    p.run(K, V, stack_layers(wl, host, [1, 2], "Q"))
    c = SpindleKVPagedCache(2, 2, 8, 2, 128, 64, 12, 32, "int8")
    p.store_paged(K, V, c)
    assert c.status() == 0
    r = ref_of(c)
    keep = p.keep_idx.cpu().numpy()
    fresh = R.RefCache(*(np.zeros_like(x) for x in (r.codes["k"], r.codes["v"], r.scale["k"], r.scale["v"], r.ref, r.pages, r.lens)), "int8")
    fresh.pages[:] = -1
    start = fresh.resize(p.kept_lens.cpu().numpy())
    fresh.append(start, f64(K[1:]), f64(V[1:]), keep, 700)
    same_state(c, fresh)
    # against the kept rows themselves: rounding moves a value by half a step of its block's scale at most
    for l in range(2):
        for s in range(2):
            n = int(fresh.lens[l, s])
            for g, kept in (("k", p.K_kept), ("v", p.V_kept)):
                step = np.repeat(fresh.scale[g][fresh.pages[l, s, :fresh.count(n)]].transpose(1, 0, 2).reshape(2, -1), 16, 1)[:, :n, None]
                assert (np.abs(fresh.rows(g, l, s)[0] - f64(kept[l, s, :, :n])) <= 0.5 * step).all()
    select = SpindleKVBeamSelect(1, 2, 1000)
    rng = np.random.default_rng(2)
    score = torch.zeros(2, device="cuda")
    for step in range(20):
        r = fresh
        logits = torch.from_numpy(rng.standard_normal((2, 1000)).astype(np.float32)).cuda()
        new_score, parent, _ = select.run(logits, score)
        want = R.beam(f64(logits), f64(score), 2, 2)
        assert np.array_equal(parent.cpu().numpy(), want[1])
        score = new_score.view(-1).clone()
        c.fork(parent.view(-1))
        assert r.fork(want[1][0].tolist())
        c.resize(add=1)
        at = r.resize(r.lens + 1)
        k1, v1, q = (rows((2, 2, n, 1, 128), "bf16", 3 * step + i, 0.2) for i, n in enumerate((2, 2, 8)))
        outs = []
        for l in range(2):
            c.append(k1[l:l + 1], v1[l:l + 1], layer=l)
            outs.append(c.attend(q[l:l + 1], layer=l, max_len=230).clone())
        r.append(at, f64(k1), f64(v1))
        check_attention(c, r, q, torch.cat(outs), "bf16")
    assert c.status() == 0
    same_state(c, r)


def test_storing_a_prompt_refuses_before_it_gives_anything_back():
    from gpu_util import generate, make_config, stack_layers, torch_dtype
    from paper_2507_06517_b200 import synth
    from paper_2507_06517_b200.pipeline import SpindleKVPagedCache, SpindleKVPass
    wl = synth.Workload("paged", 3, 1, 8, 2, 128, "bf16", 32, (300, 300), 40, (0.05, 0.3), 4, "recency", budget_tokens=100.0, seed=4)
    host = generate(wl)
    p = SpindleKVPass(make_config(wl), wl.seq_lens, torch_dtype(wl))
    K, V = (stack_layers(wl, host, [0, 1, 2], x) for x in "KV")
    p.run(K, V, stack_layers(wl, host, [1, 2], "Q"))
    c = SpindleKVPagedCache(2, 2, 8, 2, 128, 64, 12, 32, "int8")
    p.store_paged(K, V, c)
    r = ref_of(c)
    for k, v in ((K[:, :1], V[:, :1]), (K[..., :200, :], V[..., :200, :]), (K[:1], V[:1]), (K, V[:, :, :1]), (K, V.cpu())):
        with pytest.raises(ValueError):
            p.store_paged(k, v, c)
    with pytest.raises(ValueError):
        p.store_paged(K, V, SpindleKVPagedCache(2, 3, 8, 2, 128, 64, 12, 32, "int8"))
    same_state(c, r)
    # once more over what it holds: the same content again
    p.store_paged(K, V, c)
    again = ref_of(c)
    assert c.status() == 0 and np.array_equal(again.lens, r.lens)
    for l, s in r.units():
        for g in "kv":
            assert np.array_equal(again.rows(g, l, s)[0], r.rows(g, l, s)[0])


@pytest.mark.parametrize("n_rows", [1, 4])
@pytest.mark.parametrize("given_back", [False, True])
def test_first_attention_of_a_cache_on_a_stream_beside_a_busy_one(n_rows, given_back):
    # the very first call goes to a side stream while the current one is far behind: nothing that the call needs may be in its queue
    c = make(1, 2, 16, 2, 128, 400, 160, 32, "int8")
    r = fill(c, [[5000, 3000]], spread=0.3)
    q = rows((1, 2, 16, n_rows, 128), "bf16", 5, 0.2)
    if given_back:
        c.ws_attend = None
    make(1, 1, 16, 2, 128, 4, 2, 32, "int8").attend(torch.zeros_like(q[:, :1]))        # kernels are loaded
    scratch, side = torch.full((64 << 20,), 3.0, device="cuda"), torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), torch.empty(1 << 18, dtype=torch.uint8, device="cuda")      # blocks to hand out
    side.wait_stream(torch.cuda.current_stream())
    free = torch.full((q.numel(),), 7.0, dtype=q.dtype, device="cuda")
    for _ in range(100):
        scratch.mul_(1.0001)
    free.fill_(9.0)
    del free                                   # a block that the current stream has still to write
    out = c.attend(q, stream=side)
    with torch.cuda.stream(side):
        got = out.cpu()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), got)         # and what it did afterwards changed nothing
    check_attention(c, r, q, out, "bf16")
    assert c.status() == 0


@pytest.fixture
def limits():
    from paper_2507_06517_b200 import binding as B
    yield B.spindlekv_set_tuning
    for k in range(5):
        B.spindlekv_set_tuning(k, -1)


# which kernel serves a call: a block per unit, runs of the kernel for few columns (one, two and four column tiles), tiles of 32, 64, 128.
# The hints make runs long enough that block 3 has tokens
SHORT, LONG = [[40, 100, 33], [7, 0, 90]], [[9000, 700, 1], [0, 900, 8000]]
GIVE_UP = [("bf16", 64, 2, 1, SHORT, 128), ("f32", 128, 4, 1, SHORT, 128), ("bf16", 128, 4, 1, LONG, 700), ("f32", 128, 8, 2, LONG, 700),
           ("bf16", 64, 8, 4, LONG, 700), ("bf16", 128, 8, 4, LONG, 520), ("bf16", 128, 8, 8, LONG, 520), ("bf16", 128, 8, 16, LONG, 9000)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,hn,n_rows,lens,max_len", GIVE_UP)
def test_a_wait_that_runs_out_comes_back_with_a_status(limits, dtype, d, hn, n_rows, lens, max_len, fmt):
    # a block waits, with a short bound, for keys that nobody has asked for: the call returns and says so, and the next one is as ever
    from paper_2507_06517_b200 import binding as B
    c = make(2, 3, 2 * hn, 2, d, 700, 300, 32, fmt)
    r = fill(c, lens, dtype, spread=0.3)
    q = rows((2, 3, 2 * hn, n_rows, d), dtype, 5, 0.2)
    limits(B.TUNE_MBAR_WAIT_CYCLES, 2_000_000)
    limits(B.TUNE_PAGED_WITHHOLD, 3)
    out = torch.full_like(q, 7.0)
    c.attend(q, out=out, max_len=max_len)
    assert c.status() == B.TIMEOUT
    limits(B.TUNE_PAGED_WITHHOLD, -1)
    c.attend(q, out=out, max_len=max_len)
    assert c.status() == B.OK
    check_attention(c, r, q, out, dtype)


def test_status_of_a_call_with_a_block_per_unit_is_the_last_blocks(limits):
    # whichever block gives up, and whatever the workspace held: nobody's OK may cover it, and nothing of it stays
    from paper_2507_06517_b200 import binding as B
    from paper_2507_06517_b200.pipeline import record_graph
    c = make(3, 20, 4, 2, 64, 3 * 20 * 8, 8, 16, "int8")
    lens = np.random.default_rng(1).integers(0, 129, (3, 20))
    lens[0, 0], lens[2, 19], lens[1, 3] = 5, 128, 0
    r = fill(c, lens.tolist(), spread=0.3)
    q = rows((3, 20, 4, 1, 64), "bf16", 5, 0.2)
    limits(B.TUNE_MBAR_WAIT_CYCLES, 2_000_000)
    for block in (119, 0):                     # the last unit's, and the first one's
        limits(B.TUNE_PAGED_WITHHOLD, block)
        c.ws_attend.random_(0, 256)
        c.attend(q, max_len=128)
        assert c.status() == B.TIMEOUT
        limits(B.TUNE_PAGED_WITHHOLD, -1)
        for _ in range(2):
            check_attention(c, r, q, c.attend(q, max_len=128), "bf16")
            assert c.status() == B.OK
    graph = record_graph(lambda: c.attend(q, max_len=128))
    for _ in range(3):
        c.ws_attend.random_(0, 256)
        graph.replay()
        graph.replay()
        assert c.status() == B.OK


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n_rows", [4, 8, 16])
def test_attention_of_many_columns_that_begins_with_missing_pages(fmt, n_rows):
    # scores near -200 (in powers of two): a column's reference is that of the tokens it sees, however many tiles of nothing come first
    c = make(1, 12, 16, 2, 128, 12 * 50, 50, 64, fmt)
    r = ref_of(c)
    lens = 3200 - 37 * np.arange(12)[None]
    start = r.resize(lens)
    c.resize(lens_t(lens))
    K, V = rows((1, 12, 2, 3200, 128), "bf16", 1, 0.1), rows((1, 12, 2, 3200, 128), "bf16", 2, 0.3)
    K[..., 0] = -40
    for s in range(12):
        V[0, s, :, 128 * (s % 4):128 * (s % 4) + 128] = 0     # the first tile that is seen has a say in the weights' sum alone
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    for s in range(12):
        c.pages[0, s, :2 * (s % 4)] = -1                      # none, one, two, three tiles at the front
        c.pages[0, s, 8 + s:8 + s + s % 7] = 1 << 20          # and some inside, where a run may begin
    c.pages[0, 11] = -1                                       # nothing at all
    q = rows((1, 12, 16, n_rows, 128), "bf16", 5, 0.2)
    q[..., 0] = 40
    out = torch.full_like(q, 7.0)
    c.attend(q, out=out)
    check_attention(c, ref_of(c), q, out, "bf16")
    assert (out[0, 11] == 0).all() and c.status() == 0


def check_rows(c, r, q, out, dtype):
    """As ``check_attention``, row by row from what the row sees: |error| <= half a step of the output, plus, per token that has a weight at all
    (2^-100 of the row's largest one: below that it adds nothing to a float64 sum either), its weight's relative error (2^-12 in one fp16
    piece, 2^-22 in two; twice the score's) and half of fp16's smallest step.  That step is 2^-24, of a weight times 128 times the block's
    scale in units of a power of two that is at most 2^8 (and the power's factor of two) above the scale where one piece holds both: 2^-23 of
    the token's value; two pieces hold the weight alone: 2^-31.  Rows that see a block into which an infinity was written are NaN."""
    got, x = f64(out), f64(q)
    hn, n_rows = x.shape[2] // r.heads, x.shape[3]
    half, weight, step = (2.0 ** -8, 2.0 ** -12, 2.0 ** -23) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -22, 2.0 ** -31)
    for l, s in r.units():
        k, v = r.rows("k", l, s)[0], r.rows("v", l, s)[0]
        for h in range(x.shape[2]):
            kk, vv = k[h // hn], v[h // hn]
            for i in range(n_rows):
                n = max(kk.shape[0] - n_rows + 1 + i, 0)
                if n == 0:
                    assert (got[l, s, h, i] == 0).all()
                    continue
                if np.isnan(vv[:n]).any():
                    assert np.isnan(got[l, s, h, i]).all()
                    continue
                y = kk[:n] @ x[l, s, h, i] / np.sqrt(c.d)
                w = np.exp(y - y.max())
                w /= w.sum()
                has = w > 2.0 ** -100 * w.max()
                want, mag = w @ vv[:n], w @ np.abs(vv[:n])
                top = (np.abs(kk[:n][has]) @ np.abs(x[l, s, h, i])).max() / np.sqrt(c.d)
                err = ((c.d + 16) * 2.0 ** -23 + (0 if dtype == "bf16" else 2.0 ** -22)) * top + 2.0 ** -20
                bound = half * np.abs(want) + 1.01 * mag * (weight + 2 * err) + step * w.max() * np.abs(vv[:n][has]).sum(0)
                assert np.isfinite(got[l, s, h, i]).all()
                worst = (np.abs(got[l, s, h, i] - want) / np.maximum(bound, 1e-300)).max()
                assert worst <= 1, (l, s, h, i, worst)


UNEVEN = [("bf16", 128, 1, 1), ("bf16", 128, 8, 2), ("bf16", 128, 8, 4), ("bf16", 128, 8, 8), ("bf16", 128, 8, 16), ("bf16", 64, 1, 2), ("bf16", 64, 8, 4),
          ("f32", 128, 1, 2), ("f32", 128, 8, 2), ("f32", 64, 8, 4)]


def uneven_cache(fmt, d, dtype, n, n_seqs=8):
    """Two KV heads and sequences enough for runs of several tiles.  Scores are small but for a query channel that tells tokens apart."""
    c = make(1, n_seqs, None, 2, d, n_seqs * (n // 64 + 1), n // 64 + 1, 64, fmt)
    r = ref_of(c)
    start = r.resize(np.full((1, n_seqs), n))
    c.resize(lens_t([[n] * n_seqs]))
    return c, r, start, rows((1, n_seqs, 2, n, d), dtype, 1, 0.1) * 0.5, rows((1, n_seqs, 2, n, d), dtype, 2, 0.1)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,hn,n_rows", UNEVEN)
def test_attention_is_untouched_by_a_large_value_that_has_no_weight(fmt, dtype, d, hn, n_rows):
    # one token, of every size, whose score is far below all others, early and late; its neighbours' codes are zeros, all other blocks count
    c, r, start, K, V = uneven_cache(fmt, d, dtype, 2500)
    for s, (at, size) in enumerate([(3, 2.0 ** 12), (3, 2.0 ** 26), (130, 2.0 ** 40), (700, 2.0 ** 30), (1280, 2.0 ** 60), (2499, 2.0 ** 40), (5, 2.0 ** 100), (64, 2.0 ** -60)]):
        V[0, s, :, at] *= size
        if size > 1:
            K[0, s, :, at] = 0
            K[0, s, :, at, 0] = -30000
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 8, 2 * hn, n_rows, d), dtype, 5, 0.2)
    q[..., 0] = q[..., 0].abs() + 1
    out = c.attend(q, max_len=100000)
    check_rows(c, r, q, out, dtype)
    assert torch.equal(out.clone(), c.attend(q, max_len=100000)) and c.status() == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,hn,n_rows", [x for x in UNEVEN if x[3] > 1])
def test_attention_is_untouched_by_values_that_a_row_does_not_see(fmt, dtype, d, hn, n_rows):
    # the newest token's value is large: rows before it are what they are without it
    c, r, start, K, V = uneven_cache(fmt, d, dtype, 2500)
    clean = V.clone()
    for s in range(8):
        V[0, s, :, -1] *= 2.0 ** (14 * s)
    q = rows((1, 8, 2 * hn, n_rows, d), dtype, 5, 0.2)
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    check_rows(c, r, q, c.attend(q, max_len=100000), dtype)
    # with the same codes where the rows look: a block of its own for the large value
    keep = torch.full((1, 8), 2496, dtype=torch.int32, device="cuda")
    c.append(K, clean, start=torch.zeros((1, 8), dtype=torch.int32, device="cuda"))
    c.append(K[:, :, :, 2496:].contiguous(), torch.cat([clean[:, :, :, 2496:2499], V[:, :, :, 2499:]], 3), start=keep)
    r = ref_of(c)
    check_rows(c, r, q, c.attend(q, max_len=100000), dtype)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,hn,n_rows", UNEVEN)
def test_attention_over_blocks_of_every_size(fmt, dtype, d, hn, n_rows):
    # values of sizes from 2^-60 to 2^60, block by block, in patterns that repeat inside a tile, rise, fall, and leave blocks of zeros; the
    # weight lies on one size of blocks after the other.  The last pattern rises beyond the types' range: infinities
    c, r, start, K, V = uneven_cache(fmt, d, dtype, 2500)
    block = torch.arange(2500, device="cuda") // 16
    sizes = [block % 8 * 12 - 40, block % 2 * 20, block // 8 * 6 - 60, 60 - block // 8 * 6, block * 7919 % 120 - 60, block % 3 * -9, (block == 40) * 60, block % 157]
    for s, e in enumerate(sizes):
        V[0, s] = (V[0, s].float() * torch.exp2(e.float())[:, None]).to(V.dtype)
        K[0, s, :, :, 0] = -(e.float() * (s % 3) * 0.5).to(K.dtype)      # the larger the value, the less it counts: not, a little, in full
    V[0, 4, :, 160:192] = 0
    V[0, 5, :, 0:128] = 0
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 8, 2 * hn, n_rows, d), dtype, 5, 0.2) * 0.3
    q[..., 0] = 2 * np.sqrt(d) * np.log(2)                               # a score falls by s % 3 powers of two for every power of the value
    check_rows(c, r, q, c.attend(q, max_len=100000), dtype)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,hn,n_rows", UNEVEN + [("bf16", 64, 3, 1), ("bf16", 128, 8, 1), ("f32", 128, 8, 4)])
def test_attention_over_keys_with_outlier_channels(fmt, dtype, d, hn, n_rows):
    """Three channels forty times the size of the others, which the queries leave alone: most codes are small.  int8 keys may enter the products with
    128 added and have it taken off again: the d + 16 roundings of a score (2^-23 each) are then relative to sum |q_i| (|k_i| + 128 steps of
    the block's scale) in place of sum |q_i k_i|.  A weight is off by that and by 2^-20 of the power function, twice over, and by its own
    rounding, to half of fp16's smallest step at worst (``check_rows``; the largest weight is at most 1); a bf16 result by 2^-8 of itself."""
    c, r, start, K, V = uneven_cache(fmt, d, dtype, 1500, n_seqs=3)
    K *= 2
    K[..., [5, d // 2, d - 1]] *= 40
    c.append(K, V)
    r.append(start, f64(K), f64(V))
    q = rows((1, 3, 2 * hn, n_rows, d), dtype, 5, 0.2)
    q[..., [5, d // 2, d - 1]] = 0
    got, x = f64(c.attend(q)), f64(q)
    want, mag, top = r.attend(x)
    steps = max(r.scale["k"][p].max() for l, s in r.units() for p in r.pages[l, s, :r.count(r.lens[l, s])])
    offset = 128 * steps * np.abs(x).sum(-1) / np.sqrt(d) if fmt == "int8" else 0 * top
    assert fmt != "int8" or (offset > 64 * top).any()
    err = (d + 16) * 2.0 ** -23 * (top + offset) + (0 if dtype == "bf16" else 2.0 ** -22 * top) + 2.0 ** -20
    half, weight, step = (2.0 ** -8, 2.0 ** -12, 2.0 ** -23) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -22, 2.0 ** -31)
    big = max(np.abs(r.rows("v", l, s)[0]).max() for l, s in r.units())
    bound = half * np.abs(want) + 1.01 * mag * (weight + 2 * err[..., None]) + step * 1500 * big
    assert (np.abs(got - want) <= bound).all()
    # and far inside that where no bound says so: rounding errors of both signs
    assert np.sqrt(((got - want) ** 2).mean() / (want ** 2).mean()) < (2.0 ** -8 if dtype == "bf16" else 2.0 ** -16)


@pytest.mark.parametrize("n_rows,hn", [(3, 8), (7, 8), (16, 8)])
@pytest.mark.parametrize("n_layers,n_seqs", [(3, 41), (1, 740)])
def test_attention_of_many_columns_over_many_sequences(n_layers, n_seqs, n_rows, hn):
    # more sequences than lanes, and than threads; many of them empty or shorter than the new rows
    c = make(n_layers, n_seqs, hn, 1, 128, n_layers * n_seqs * 6, 22, 32, "int8")
    rng = np.random.default_rng(n_seqs + n_rows)
    lens = np.where(rng.random((n_layers, n_seqs)) < 0.4, 0, rng.integers(1, 60, (n_layers, n_seqs)))
    lens[rng.random((n_layers, n_seqs)) < 0.08] = 290
    lens[-1, -1] = 700
    r = fill(c, lens.tolist(), spread=0.3)
    q = rows((n_layers, n_seqs, hn, n_rows, 128), "bf16", 5, 0.2)
    out = torch.full_like(q, 7.0)
    c.attend(q, out=out)
    check_attention(c, r, q, out, "bf16")
    assert c.status() == 0


def test_page_operators_over_a_large_pool():
    # the planning block walks more than one stretch of 32768 pages: free pages, holes and live pages beyond the first
    n = 70001
    c = make(2, 5, 2, 1, 64, n, 300, 16, "int8")
    rng = np.random.default_rng(3)
    taken = np.sort(rng.choice(n, 69000, replace=False))
    held = torch.zeros(n, dtype=torch.int32)
    held[torch.from_numpy(taken)] = 1                     # pages that another table holds
    c.page_ref.copy_(held)
    r = fill(c, [[4800, 37, 0, 16, 1000], [3000, 1, 5, 700, 99]])
    same_state(c, r)
    c.page_ref.sub_(held.cuda())                          # that table is gone: holes everywhere
    r = ref_of(c)
    assert int(c.compact()) == r.compact()
    same_state(c, r)
    assert r.fork([0, 0, 1, 0, 4])
    c.fork(lens_t([0, 0, 1, 0, 4]))
    same_state(c, r)
    for lens in ([[4790, 4800, 30, 100, 999], [0, 3000, 0, 2990, 105]], [[0] * 5] * 2):
        start = r.resize(np.array(lens))
        assert start is not None
        c.resize(lens_t(lens))
        assert c.status() == 0 and np.array_equal(c.start.cpu().numpy(), start)
        for what in ("ref", "lens", "pages"):
            assert np.array_equal(getattr(ref_of(c), what), getattr(r, what)), what


def test_fork_of_as_many_sequences_as_there_may_be():
    c = make(1, 1024, 2, 1, 64, 6000, 6, 16, "e4m3")
    rng = np.random.default_rng(1)
    r = fill(c, rng.integers(0, 60, (1, 1024)).tolist())
    parent = rng.integers(-1, 1024, 1024)
    assert r.fork(parent)
    c.fork(lens_t(parent))
    assert c.status() == 0
    same_state(c, r)
