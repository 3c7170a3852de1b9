"""What rows that come behind a token in its block of 16 do to it: they may raise the block's scale, and its codes are rounded to that.

Under a scale s a code of 2^-6 s or more has four significant bits whatever s is, so a number that was stored under a smaller scale stays what it was; below that codes are steps of 2^-9 s, and the number moves by half of one at
most, 2^-10 s.  s is the smallest power of two with amax <= 448 s, so s < amax / 224 (or 2^-100): less than 2^-17 of the largest number.  An output is a mean of values and moves by no more,
beside its rounding and the arithmetic's part of the bound of tests/test_gpu_kv8.py, once on each side."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Setup, pv  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("outlier", [1.0, 2.0 ** 5, 2.0 ** 10, 2.0 ** 14, 2.0 ** 20])
def test_a_rejected_row_moves_its_block_by_a_half_step(pv, rows, outlier):  # noqa: F811
    alone, joined = (Setup(pv, [69], [rows + 1], heads=2, hd=64, seed=3) for _ in range(2))
    k, v = alone.draw(69, "bf16"), alone.draw(69, "bf16")
    nk, nv = alone.draw(rows + 1, "bf16"), alone.draw(rows + 1, "bf16")
    nv[rows] = (nv[rows].float() * outlier).to(nv.dtype)
    q = torch.from_numpy(alone.r.normal(size=(rows + 1, 4, 64))).to(torch.bfloat16).cuda()
    for s in (alone, joined):
        s.pool.append(s.seqs([0, 69], [0]), k.cuda(), v.cuda())
    first = lambda s: s.pool.read(s.seqs([0, 69 + rows], [0]), 69 + rows, dtype=torch.float32)  # noqa: E731
    alone.pool.append(alone.seqs([0, rows]), nk[:rows].cuda(), nv[:rows].cuda())
    joined.pool.append(joined.seqs(), nk.cuda(), nv.cuda())
    (ak, av), (jk, jv) = first(alone), first(joined)
    assert torch.equal(ak[:64], jk[:64]) and torch.equal(av[:64], jv[:64])                    # other blocks: nothing moves
    amax = torch.cat([v[64:], nv]).float().abs().amax((0, 2)).cuda()
    s = 2.0 ** torch.ceil(torch.log2(amax / 448)).view(1, -1, 1)
    assert ((av[64:] - jv[64:]).abs() <= 2.0 ** -10 * s).all()
    kept = av[64:].abs() >= 2.0 ** -6 * s
    assert torch.equal(av[64:][kept], jv[64:][kept])
    a, j = alone.pool.attention(alone.seqs([0, rows]), q[:rows]).float(), joined.pool.attention(joined.seqs(), q).float()[:rows]
    mag = av.abs().amax((0, 2)).repeat_interleave(2).view(1, -1, 1)
    moved = (2.0 ** -10 * s).view(-1).repeat_interleave(2).view(1, -1, 1)
    assert ((a - j).abs() <= moved + 2.0 ** -8 * torch.maximum(a.abs(), j.abs()) + 2 * (2.0 ** -12 + 2.0 ** -11) * mag).all()
    if outlier == 1.0:
        assert (jv[64:] == av[64:]).float().mean() > 0.99
