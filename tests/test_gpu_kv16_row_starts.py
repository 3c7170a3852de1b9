"""Entries of row_start from which the difference of two wraps: such a sequence has no rows, the others what they have."""
import numpy as np
import pytest
import torch

from test_gpu_kv16 import Setup, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu

LOW = -2 ** 31


@pytest.mark.parametrize("start", [[5, LOW, 3], [12, LOW + 648, LOW], [1, LOW, LOW + 1]])
@pytest.mark.parametrize("reach", [16, 1 << 17])                          # (few rows a tile, and many)
def test_cache(pv, start, reach):  # noqa: F811
    s = Setup(pv, [20, 30], [6, 6], heads=2, hd=64)
    s.fill_prefix()
    s.fill_rows()
    tables = np.concatenate([s.tables, np.full((2, max(0, reach // 16 - s.tables.shape[1])), -1, np.int32)], axis=1)
    wild, before = s.seqs(start=start, tables=tables), torch.nan_to_num(s.pool.pages)
    k, q = s.draw(12).cuda(), torch.randn(12, 20, 64, device="cuda").bfloat16()
    turned = torch.full_like(q, 7.0)
    s.pool.append(wild, k, k, rotary=pv.Rotary(64), q=q, q_out=turned)
    s.pool.keep(wild, torch.arange(1, 13, dtype=torch.int32, device="cuda"), dev([5, 5]))
    assert (turned == 7).all() and torch.equal(torch.nan_to_num(s.pool.pages), before)
    for mask in (None, torch.ones(12, 3, dtype=torch.int64, device="cuda")):
        out, lse = torch.full_like(q, 7.0), torch.full((12, 20), 7.0, device="cuda")
        s.pool.attention(wild, q, mask=mask, out=out, lse=lse)
        assert (out == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_verification(pv, kind, temperature):  # noqa: F811
    x, tokens, u = torch.randn(12, 5000, device="cuda"), dev(np.arange(12)), torch.rand(12, 2, device="cuda")
    more = {"drawn": {"draft_probs": torch.softmax(x, 1)}, "given": {}, "tree": {"parent": dev(np.maximum(np.arange(12) - 1, 0))}}[kind]
    for start in ([5, LOW, 3], [12, LOW + 648, LOW]):
        got = pv.verify_drafts(dev(start), x, tokens, u, temperature=temperature, **more)
        assert got.accepted.tolist() == [0, 0] and got.next_token.tolist() == [-1, -1] and not got.probs.any()
        assert got.path is None or (got.path == -1).all()
