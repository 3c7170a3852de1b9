"""The operators have no forward-mode derivatives either: tensors that carry a tangent are refused, not answered without one."""
import pytest
import torch
from torch.autograd import forward_ad

import test_gpu_kv8
from test_gpu_kv16 import Setup, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu


def test_tensors_with_tangents(pv):  # noqa: F811
    s, old = Setup(pv, [20], [3], heads=2, hd=64), test_gpu_kv8.Setup(pv, [20], [3], heads=2, hd=64)
    s.fill_prefix(), old.fill_prefix()
    k, v, q, p = s.draw(3).cuda(), s.draw(3).cuda(), torch.randn(3, 4, 64, device="cuda").bfloat16(), dev([0, 1, 2])
    rot = pv.Rotary(64)
    s.pool.append(s.seqs(), k, v), old.pool.append(old.seqs(), k, v)
    x, u, tokens, begin = torch.randn(3, 100, device="cuda"), torch.rand(3, 2, device="cuda"), dev([1, 2, 3]), dev([0, 3])
    probs, hot, lse = torch.softmax(x, 1), torch.ones(1, device="cuda"), torch.zeros(3, 4, device="cuda")
    pages, codes = torch.nan_to_num(s.pool.pages).clone(), old.pool.codes.clone()
    want = s.pool.attention(s.seqs(), q)
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        calls = [lambda: s.pool.append(s.seqs(), dual(k), v), lambda: s.pool.append(s.seqs(), k, dual(v)), lambda: s.pool.append(s.seqs(), k, v, rotary=rot, q=dual(q)),
                 lambda: s.pool.append(s.seqs(), k, v, rotary=rot, q=q, q_out=dual(q)), lambda: rot.rotate(dual(q), p), lambda: rot.rotate(q, p, out=dual(q)), lambda: s.pool.attention(s.seqs(), dual(q)),
                 lambda: s.pool.attention(s.seqs(), dual(q)[:, :2]), lambda: s.pool.attention(s.seqs(), q, out=dual(q)), lambda: s.pool.attention(s.seqs(), q, lse=dual(lse)),
                 lambda: s.pool.attention(s.seqs(), dual(q), stream=torch.cuda.Stream()), lambda: pv.verify_drafts(begin, dual(x), tokens, u), lambda: pv.verify_drafts(begin, x, tokens, dual(u)),
                 lambda: pv.verify_drafts(begin, x, tokens, u, draft_probs=dual(probs)), lambda: pv.verify_drafts(begin, x, tokens, u, temperature=dual(hot)),
                 lambda: pv.KV16Pool(4, 2, 64, pages=dual(torch.zeros(4, 2, 2, 1024, dtype=torch.bfloat16, device="cuda"))),
                 lambda: old.pool.append(old.seqs(), dual(k), v), lambda: old.pool.append(old.seqs(), k, dual(v)), lambda: old.pool.attention(old.seqs(), dual(q)),
                 lambda: old.pool.attention(old.seqs(), q, out=dual(q)), lambda: old.pool.attention(old.seqs(), q, lse=dual(lse)), lambda: old.pool.read(old.seqs(), 3, out=(dual(k), k)),
                 lambda: pv.token_logprobs(dual(x), None, top=2)]
        for i, call in enumerate(calls):
            with pytest.raises(pv.PVError, match="gradient"):
                call()
                pytest.fail(f"call {i} went through")
            with torch.no_grad(), pytest.raises(pv.PVError, match="gradient"):      # (which leaves forward mode as it is)
                call()
        # what carries none is taken, and where derivatives are off altogether
        assert torch.equal(s.pool.attention(s.seqs(), q), want) and torch.equal(s.pool.attention(s.seqs(), forward_ad.unpack_dual(dual(q)).primal), want)
        d = dual(q)
        with torch.inference_mode():
            assert torch.equal(s.pool.attention(s.seqs(), d), want)
    assert torch.equal(torch.nan_to_num(s.pool.pages), pages) and torch.equal(old.pool.codes, codes)


def test_inside_a_jvp(pv):  # noqa: F811
    s = Setup(pv, [20], [3], heads=2, hd=64)
    s.fill_prefix(), s.fill_rows()
    q, seqs = torch.randn(3, 4, 64, device="cuda").bfloat16(), s.seqs()
    with pytest.raises(pv.PVError, match="gradient"):
        torch.func.jvp(lambda y: s.pool.attention(seqs, y), (q,), (torch.ones_like(q),))


def test_frequencies_that_require_a_gradient(pv):  # noqa: F811
    """A Rotary keeps them: refused when it is made, whatever the mode."""
    turns = torch.rand(32, dtype=torch.float64, device="cuda")
    pv.Rotary(64, turns=turns)
    with forward_ad.dual_level(), pytest.raises(pv.PVError, match="gradient"):
        pv.Rotary(64, turns=forward_ad.make_dual(turns, turns))
    turns.requires_grad_()
    with pytest.raises(pv.PVError, match="gradient"):
        pv.Rotary(64, turns=turns)
    with torch.no_grad(), pytest.raises(pv.PVError, match="gradient"):
        pv.Rotary(64, turns=turns)
