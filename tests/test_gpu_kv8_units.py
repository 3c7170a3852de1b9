"""Attention over values whose blocks' scales lie far apart, under weights that all count: blocks of zeros (which have the smallest scale there is) and of small numbers among large ones.

Keys of zeros give every key the same weight, so that a row's output is the sum of the values it sees over their number.  The bound is that of tests/test_gpu_kv8.py: half a step of the output, and
2^-12 (f16) or 2^-12 + 2^-11 (bf16) of the sum of weight * |value|."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Setup, check_attention, pv  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def even(pv, n, rows, value, small, heads, dtype, room=0, pt=16):
    """n tokens of `value` (a number that a code stands for), those of the block indexes in `small` with their own; all keys zero."""
    pages = -(-(n + rows) // pt)
    pool = pv.KV8Pool(pages, heads, 64, pt)
    per = torch.full((n + rows,), float(value), dtype=torch.float64)
    for b, x in small.items():
        per[16 * b:16 * b + 16] = x
    v = per.to(torch.bfloat16).cuda().view(-1, 1, 1).expand(-1, heads, 64).contiguous()
    table = torch.cat([torch.arange(pages), torch.full((room,), -1)]).to(torch.int32).view(1, -1).cuda()
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool.append(pv.KV8Seqs(i(0, n + rows), i(0), table), torch.zeros_like(v), v)
    q = torch.randn(rows, heads * 2, 64, device="cuda").to(TYPES[dtype])
    out, lse = pool.attention(pv.KV8Seqs(i(0, rows), i(n), table), q, return_lse=True)
    seen = torch.arange(n + 1, n + rows + 1, dtype=torch.float64)
    want, mag = per.cumsum(0)[n:] / seen, per.abs().cumsum(0)[n:] / seen
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    eps = torch.finfo(TYPES[dtype]).eps / 2
    bound = eps * want.abs() + (2.0 ** -12 + (2.0 ** -11 if dtype == "bf16" else 0.0)) * mag + torch.finfo(TYPES[dtype]).tiny
    assert ((got - want.view(-1, 1, 1)).abs() <= bound.view(-1, 1, 1)).all(), (got - want.view(-1, 1, 1)).abs().max()
    assert ((lse.double().cpu() - seen.log().view(-1, 1)).abs() <= 2.0 ** -14 + 2.0 ** -22 * seen.log().view(-1, 1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 10, 40, 130])
@pytest.mark.parametrize("value,n,heads", [(288, 64, 1), (288, 1000, 2), (104, 1000, 2), (16, 3000, 64)])
@pytest.mark.parametrize("room", [0, 1250])
def test_a_block_of_zeros_behind_large_values(pv, value, n, heads, rows, dtype, room):  # noqa: F811
    even(pv, n, rows, value, {n // 16 - 1: 0.0}, heads, dtype, room)


@pytest.mark.parametrize("rows", [1, 10, 130])
def test_a_block_of_zeros_behind_thousands_of_ones(pv, rows):  # noqa: F811
    """So many heads that a workgroup has all keys of a row."""
    even(pv, 9008, rows, 1, {562: 0.0}, 256, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 40, 130])
def test_blocks_of_zeros_and_of_small_numbers_all_along(pv, rows, dtype):  # noqa: F811
    """Scales that fall step by step, 2^20 at a time, and rise again."""
    n = 1600
    small = {b: (0.0, 26 * 2.0 ** -20, 26 * 2.0 ** -40, 26 * 2.0 ** -60, 26 * 2.0 ** -80)[b % 5] for b in range(n // 16) if b % 7}
    even(pv, n, rows, 208, small, 4, dtype, 400)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 10, 40, 130])
def test_zeros_among_ordinary_numbers(pv, rows, dtype):  # noqa: F811
    s = Setup(pv, [330], [rows], heads=1, hd=128)
    n = 330 + rows
    k, v = s.draw(n, "bf16", 0.5), s.draw(n, "bf16", 3)
    for b in (0, 2, 3, 9, 14, 15, 16, 17):
        v[16 * b:16 * b + 16] = 0
    s.pool.append(s.seqs([0, n], [0]), k.cuda(), v.cuda())
    s.ref.append([0, n], [0], s.tables, k.double().numpy(), v.double().numpy())
    q = torch.from_numpy(s.r.normal(size=(rows, 4, 128))).to(TYPES[dtype])
    out, lse = s.pool.attention(s.seqs(), q.cuda(), return_lse=True)
    check_attention(s, q, out, lse)


@pytest.mark.parametrize("large_first", [False, True])
@pytest.mark.parametrize("rows", [1, 10, 40, 130])
def test_rows_that_weigh_small_values_beside_far_larger_ones(pv, rows, large_first):  # noqa: F811
    """Scales 2^60 apart; the large values' weight is e^-100 of the others', or less.  Only the weights of what counts are in the bound."""
    s = Setup(pv, [160], [rows], heads=1, hd=64)
    n = 160 + rows
    k, v = torch.zeros(n, 1, 64), torch.from_numpy(s.r.normal(size=(n, 1, 64))).float() * 2.0 ** -34
    at = slice(0, 32) if large_first else slice(80, 112)
    v[at] *= 2.0 ** 60
    k[at, 0, 0] = -28.0
    s.pool.append(s.seqs([0, n], [0]), k.cuda(), v.cuda())
    s.ref.append([0, n], [0], s.tables, k.double().numpy(), v.double().numpy())
    q = torch.from_numpy(s.r.normal(size=(rows, 6, 64))).to(torch.bfloat16)
    q[:, :, 0] = 64.0
    out, lse = s.pool.attention(s.seqs(), q.cuda(), return_lse=True)
    check_attention(s, q, out, lse)
