"""Bits of a mask name rows of the call's own sequence: those from the number of its rows on say nothing, also where the cache holds tokens there."""
import pytest
import torch

from test_gpu_kv8 import Setup, pv  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("room", [0, 1250])
@pytest.mark.parametrize("asked", [1, 4, 40])
def test_bits_behind_the_rows(pv, monkeypatch, asked, room):  # noqa: F811
    monkeypatch.setattr(Setup, "room", room)
    s = Setup(pv, [50], [60], heads=2, hd=64)
    s.fill_prefix()
    s.pool.append(s.seqs(), s.draw(60, "bf16").cuda(), s.draw(60, "bf16").cuda())
    q = torch.randn(asked, 8, 64, device="cuda", dtype=torch.bfloat16)
    bits = torch.from_numpy(s.r.integers(-2 ** 63, 2 ** 63, asked)).cuda()
    own = bits & ((1 << asked) - 1)
    seqs = s.seqs([0, asked])
    for a, b in zip(s.pool.attention(seqs, q, mask=bits, return_lse=True), s.pool.attention(seqs, q, mask=own, return_lse=True)):
        assert torch.equal(a, b)
