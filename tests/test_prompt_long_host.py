"""Scratch of prompt attention over long keys: asked for on the host, so no device is needed."""
import pytest

from paper_2507_06517_b200 import binding as B
from test_prompt_host import batch, lib


def need(keys, rows, hq, h, d, dtype=B.BF16):
    return lib.spindlekv_prompt_workspace_bytes(batch(seqs=1, most=keys), batch(seqs=1, most=rows), hq, h, d, dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_room_for_the_sums_of_long_keys(d):
    # 1200 rows of 8 heads of 4: 19 blocks of 64 positions for each head, all in one part; each SM's 256 rows have d sums and a reference
    assert need(16384, 1200, 32, 8, d) == 256
    assert need(16385, 1200, 32, 8, d) == 256 + 148 * 256 * (d + 1) * 4
    # cut into parts: the longest one counts
    cut = need(16384, 100, 32, 8, d)
    assert cut > 256 and need(16500, 100, 32, 8, d) == cut
    assert need(65536, 1, 8, 8, d) <= 512 + 37 * 8 * (d * 4 + 8)                   # few rows: parts of 2048 keys at most (32 of them; d = 64: 2 * 148 // 8), and no such sums
    assert need(1 << 20, 512, 32, 8, d) >= 2 * 512 * 32 * (d * 4 + 8) + 128 * 256 * (d + 1) * 4
