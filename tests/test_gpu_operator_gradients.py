"""The operators have no gradients: tensors that ask for one are refused, or taken as numbers where gradients are switched off."""
import pytest
import torch

from test_gpu_kv8 import Setup, pv  # noqa: F401

pytestmark = pytest.mark.gpu


def test_tensors_that_require_gradients(pv):  # noqa: F811
    s = Setup(pv, [20], [3], heads=2, hd=64)
    s.fill_prefix()
    k, v = s.draw(3, "bf16").cuda(), s.draw(3, "bf16").cuda()
    s.pool.append(s.seqs(), k, v)
    before = s.pool.codes.clone()
    q, x = torch.randn(3, 4, 64, device="cuda", dtype=torch.bfloat16), torch.randn(3, 100, device="cuda")
    want, scores = s.pool.attention(s.seqs(), q), pv.token_logprobs(x, None, top=2)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda: s.pool.append(s.seqs(), leaf(k), v), lambda: s.pool.append(s.seqs(), k, leaf(v)), lambda: s.pool.attention(s.seqs(), leaf(q)), lambda: s.pool.attention(s.seqs(), leaf(q) * 1),
             lambda: s.pool.attention(s.seqs(), q, out=leaf(q)), lambda: s.pool.attention(s.seqs(), q, lse=torch.zeros(3, 4, device="cuda", requires_grad=True)),
             lambda: s.pool.read(s.seqs(), 3, out=(leaf(k), k)), lambda: pv.token_logprobs(leaf(x), None, top=2)]
    for call in calls:
        with pytest.raises(pv.PVError, match="gradient"):
            call()
    side = torch.cuda.Stream()
    with pytest.raises(pv.PVError, match="gradient"):
        s.pool.attention(s.seqs(), leaf(q), stream=side)
    lk, lv, lq, lx = leaf(k), leaf(v), leaf(q), leaf(x)
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            s.pool.append(s.seqs(), lk, lv)
            assert torch.equal(s.pool.codes, before)
            assert torch.equal(s.pool.attention(s.seqs(), lq), want)
            assert all(torch.equal(a, b) for a, b in zip(pv.token_logprobs(lx, None, top=2), scores))
    out = s.pool.attention(s.seqs(), leaf(q).detach())
    assert torch.equal(out, want) and not out.requires_grad
