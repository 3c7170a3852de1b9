"""Values that are NaN beside pages that do not exist: rows that see such a value are NaN, whatever else the keys around it are."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Setup, check_attention, pv  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3, 16, 40, 130])
@pytest.mark.parametrize("where", ["v", "k"])
@pytest.mark.parametrize("room", [0, 1250])
def test_numbers_that_are_none_beside_missing_pages(pv, monkeypatch, rows, where, room):  # noqa: F811
    monkeypatch.setattr(Setup, "room", room)
    for token, gone in ((5, 2), (200, 13), (70, 5), (130, 0)):
        s = Setup(pv, [300], [rows], heads=2, hd=64)
        n = 300 + rows
        k, v = s.draw(n, "bf16", 0.5), s.draw(n, "bf16")
        (v if where == "v" else k)[token, 1, 9] = float("nan")
        s.pool.append(s.seqs([0, n], [0]), k.cuda(), v.cuda())
        s.ref.append([0, n], [0], s.tables, k.double().numpy(), v.double().numpy())
        t = s.tables.copy()
        t[0, gone] = -1
        for masks in (None, np.full(rows, 0x5, np.int64)):
            q = torch.from_numpy(s.r.normal(size=(rows, 4, 64))).to(torch.bfloat16)
            mask = None if masks is None else torch.from_numpy(masks).cuda()
            out, lse = s.pool.attention(s.seqs(tables=t), q.cuda(), mask=mask, return_lse=True)
            check_attention(s, q, out, lse, tables=t, masks=masks)
            assert out[:, 2:, 9].isnan().all() and not out[:, :2].isnan().any()
