"""The plain forms that the 8-bit paged cache and beam selection are tested against, pinned by hand cases."""
import numpy as np
import pytest

import paged_ref as R


def test_e4m3_code_table():
    # 1.0 is exponent 7, fraction 0; the largest number 448; the smallest 2^-9; halves to even
    assert R.decode(np.array([0x38, 0x7E, 0x01, 0xB8], np.uint8), "e4m3").tolist() == [1.0, 448.0, 2.0 ** -9, -1.0]
    x = R.decode(np.arange(127, dtype=np.uint8), "e4m3")
    assert (np.diff(x) > 0).all()
    assert R.encode(x, "e4m3").tolist() == list(range(127))
    between = (x[:-1] + x[1:]) / 2
    assert (R.encode(between, "e4m3") % 2 == 0).all()
    assert R.encode(np.array([1e9, -1e9]), "e4m3").tolist() == [0x7E, 0xFE]


def test_e4m3_codes_match_torch():
    import torch
    x = torch.randn(4096, generator=torch.Generator().manual_seed(0)) * 50
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.encode(x.double().numpy(), "e4m3"), want)


@pytest.mark.parametrize("amax,fmt,want", [(0.0, "int8", 0.0), (127.0, "int8", 1.0), (448.0, "e4m3", 1.0), (448.5, "e4m3", 2.0), (224.0, "e4m3", 0.5),
                                           (1e-44, "int8", 2.0 ** -126), (1e-44, "e4m3", 2.0 ** -126)])
def test_scales(amax, fmt, want):
    assert R.scale_of(amax, fmt) == np.float32(want)


def _cache(lens, ps=16, n_pages=12, max_pages=3, fmt="int8"):
    z = np.zeros((n_pages, 1, ps, 64), np.uint8)
    s = np.zeros((n_pages, 1, ps // 16), np.float32)
    c = R.RefCache(z, z, s, s, np.zeros(n_pages, np.int32), np.full((1, len(lens), max_pages), -1, np.int32), np.zeros((1, len(lens)), np.int32), fmt)
    assert c.resize(np.array([lens])) is not None
    return c


def test_page_operators_by_hand():
    c = _cache([20, 5])
    assert c.pages[0].tolist() == [[0, 1, -1], [2, -1, -1]] and c.ref[:4].tolist() == [1, 1, 1, 0]
    c.codes["k"][1, 0, :4] = 7
    assert c.fork([0, 0])                             # page 0 shared, page 1 the first child's, 3 its copy; 2 is free again
    assert c.pages[0].tolist() == [[0, 1, -1], [0, 3, -1]] and c.ref[:4].tolist() == [2, 1, 0, 1]
    assert (c.codes["k"][3, 0, :4] == 7).all()
    start = c.resize(np.array([[10, 20]]))            # back into the shared page: a copy of it on page 2
    assert start.tolist() == [[10, 20]] and c.pages[0, 0, 0] == 2 and c.ref[:4].tolist() == [1, 0, 1, 1]
    assert c.compact() == 3 and c.pages[0, 1].tolist()[:2] == [0, 1] and (c.codes["k"][1, 0, :4] == 7).all()
    assert not c.fork([0, 2]) and c.resize(np.array([[0, 49]])) is None


def test_attention_of_one_token_is_its_value():
    c = _cache([1], fmt="e4m3")
    c.append(np.array([[0]]), np.ones((1, 1, 1, 1, 64)), np.full((1, 1, 1, 1, 64), 2.0))
    out, mag, _ = c.attend(np.ones((1, 1, 2, 3, 64)))
    assert (out[0, 0, :, 2] == 2).all() and (out[0, 0, :, :2] == 0).all() and (mag[0, 0, :, 2] == 2).all()


def test_beam_by_hand():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]))
    s, p, t = R.beam(x, np.log([0.5, 0.5]), 2, 4)
    assert p.tolist() == [[1, 0, 0, 0]] and t.tolist() == [[1, 0, 1, 2]]      # 0.4, 0.25, then two of 0.125
    s, p, t = R.beam(x, np.log([0.5, 0.5]), 2, 2, finished=[True, False], eos=2)
    assert p.tolist() == [[0, 1]] and t.tolist() == [[2, 1]] and np.allclose(s, np.log([[0.5, 0.4]]))
