"""Attention over the 16-bit cache has the same weights whatever tile its rows come to lie in: pairs of numbers of the pool's type (tests/kv16_ref.py is the oracle).

Values that cancel leave an output next to nothing of its own rounding, so that what is left is the weights'.  A score is one product of two short numbers, exact in 32 bits, of at most 2 in magnitude; its exponent, with what is
added to it, is at most 16 and off by 2^-20 (the factor by 2^-25 of 6, the sum by half a step of 16), the exponential by 2^-23: a weight is off by 2^-19 of itself, and by its pair's 2^-16 in bf16 (half a step of half a
step, 2^-8 each), 2^-22 in f16 and 2^-32 of the largest.  Sums of up to 1800 of them in 32 bits, 16 and then 32 lanes apart, then one after the other for steps of 32 or 64: some 60 additions in a row, 60 * 2^-24 < 2^-18.  In the
numerator and in the sum: less than 2^-14.9 of sum(weight * |value|) in bf16 and 2^-16.4 in f16; asked for are 2^-14 and 2^-16, beside half a step of the output.  Weights of one number of the type, off by up to 2^-8 and 2^-11, are
several times outside on every case here."""
import numpy as np
import pytest
import torch

from test_gpu_kv16 import TYPES, dev, pv  # noqa: F401
from test_gpu_kv16_many_rows import TILES, Far

pytestmark = pytest.mark.gpu

FEW = {"16, one tile": ([40], [1], 2, 8, 16, 4096), "16, two tiles": ([100], [8], 2, 8, 16, 4096), "16, chunks": ([1700], [4], 1, 4, 16, 4096)}
CASES = {**{k: v for k, v in TILES.items() if k != "64, one head a kv head" and k != "128, one head a kv head"}, **FEW}


@pytest.mark.parametrize("case", list(CASES.values()), ids=list(CASES))
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 64)])
def test_values_that_cancel(pv, case, dtype, hd, masked):  # noqa: F811
    """Keys two by two, weights 1.6 % apart at most, with values of opposite signs."""
    s = Far(pv, case, hd, dtype)
    total = [p + w for p, w in zip(s.prefix, s.rows)]
    n = sum(total)
    k, v = torch.zeros(n, s.heads, hd), torch.zeros(n, s.heads, hd)
    half = s.r.integers(-126, 126, ((n + 1) // 2, s.heads))
    k[:, :, 0] = torch.from_numpy(np.stack([half, half + 1], 1).reshape(-1, s.heads)[:n] / 64.0).float()
    sign = s.r.integers(0, 2, ((n + 1) // 2, s.heads, hd)) * 2.0 - 1
    v[:] = torch.from_numpy(np.stack([sign, -sign], 1).reshape(-1, s.heads, hd)[:n]).float()
    s.put(np.concatenate([[0], np.cumsum(total)]).astype(np.int32), [0] * len(total), k.to(s.dtype), v.to(s.dtype))
    q = torch.zeros(s.n, s.q_heads, hd)
    q[..., 0] = torch.from_numpy(s.r.integers(32, 65, (s.n, s.q_heads)) / 64.0).float()
    q = q.to(s.dtype)
    m = s.r.integers(0, 2 ** 63, (s.n, 4)).astype(np.int64) | 1
    whole = [sum(int(w) << (64 * i) for i, w in enumerate(row.view(np.uint64))) for row in m] if masked else None
    out = s.pool.attention(s.seqs(), q.cuda(), scale=1.0, mask=dev(m, torch.int64) if masked else None).double().cpu().numpy()
    want, _, mag = s.ref.attention(s.start, s.prefix, s.tables, q.double().numpy(), 1.0, whole)
    bound = torch.finfo(s.dtype).eps / 2 * np.abs(want) + (2.0 ** -14 if dtype == "bf16" else 2.0 ** -16) * mag
    worst = (np.abs(out - want) / bound).max()
    assert worst <= 1, worst


@pytest.mark.parametrize("case", list(CASES.values()), ids=list(CASES))
@pytest.mark.parametrize("hd", [64, 128])
def test_values_up_to_where_outputs_are_sure_to_be_finite(pv, case, hd):  # noqa: F811
    """All of one sign and nearly 2^120 / tokens, scores that rise by less than results are rescaled at: sums relative to a weight 2^8 below the largest."""
    s = Far(pv, case, hd, "bf16")
    total = [p + w for p, w in zip(s.prefix, s.rows)]
    n = sum(total)
    place = np.concatenate([np.arange(m) / max(m, 2) for m in total])
    k, v = torch.zeros(n, s.heads, hd), torch.from_numpy(s.r.uniform(0.5, 0.99, (n, s.heads, hd)) * 2.0 ** 120 / max(total)).float()
    k[:, :, 0] = torch.from_numpy(np.floor(place * 5.5 * 16) / 16).float()[:, None]
    s.put(np.concatenate([[0], np.cumsum(total)]).astype(np.int32), [0] * len(total), k.to(s.dtype), v.to(s.dtype))
    q = torch.zeros(s.n, s.q_heads, hd)
    q[..., 0] = 1.0
    q = q.to(s.dtype)
    out = s.pool.attention(s.seqs(), q.cuda(), scale=1.0).double().cpu().numpy()
    want, _, mag = s.ref.attention(s.start, s.prefix, s.tables, q.double().numpy(), 1.0)
    assert np.isfinite(out).all() and (np.abs(out - want) <= torch.finfo(s.dtype).eps / 2 * np.abs(want) + 2.0 ** -14 * mag).all()
