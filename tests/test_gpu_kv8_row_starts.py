"""The 8-bit cache: entries of row_start from which the difference of two wraps.  Such a sequence has no rows, the others what they have."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Setup, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu

LOW = -2 ** 31


@pytest.mark.parametrize("start", [[5, LOW, 3], [12, LOW + 648, LOW], [1, LOW, LOW + 1]])
@pytest.mark.parametrize("reach", [16, 1 << 15])                          # (few rows a tile, and many)
@pytest.mark.parametrize("heads", [2, 20])
def test_cache(pv, start, reach, heads):  # noqa: F811
    s = Setup(pv, [20, 30], [6, 6], heads=2, hd=64)
    s.fill_prefix()
    tables = np.concatenate([s.tables, np.full((2, max(0, reach // 16 - s.tables.shape[1])), -1, np.int32)], axis=1)
    wild, codes, scales = s.seqs(start=start, tables=tables), s.pool.codes.clone(), s.pool.scales.clone()
    k, q = s.draw(12, "bf16").cuda(), torch.randn(12, heads, 64, device="cuda").bfloat16()
    s.pool.append(wild, k, k)
    assert torch.equal(s.pool.codes, codes) and torch.equal(s.pool.scales, scales)
    read = torch.full((2, 12, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda").unbind(0)
    s.pool.read(wild, 12, out=read)
    assert bool((read[0] == 7).all()) and bool((read[1] == 7).all())
    for mask in (None, torch.ones(12, dtype=torch.int64, device="cuda")):
        out, lse = torch.full_like(q, 7.0), torch.full((12, heads), 7.0, device="cuda")
        s.pool.attention(wild, q, mask=mask, out=out, lse=lse)
        assert bool((out == 7).all()) and bool((lse == 7).all())


def test_a_sequence_beside_it(pv):  # noqa: F811
    """The first one's end is the second's beginning: where that is wild the first has the rows up to it, or none, and the third what its two entries say."""
    s = Setup(pv, [20, 30, 25], [4, 4, 4], heads=2, hd=64)
    s.fill_prefix()
    q = torch.randn(12, 4, 64, device="cuda").bfloat16()
    want, got = (torch.nan_to_num(s.pool.attention(s.seqs(start=x), q, out=torch.full_like(q, 7.0))) for x in ([8, 8, 8, 12], [8, LOW, 8, 12]))      # (tokens that nobody wrote are NaN)
    same = torch.equal(got[8:], want[8:]), bool((got[8:] == 7).all())
    assert bool((want[:8] == 7).all()) and bool((got[:8] == 7).all()) and any(same)
