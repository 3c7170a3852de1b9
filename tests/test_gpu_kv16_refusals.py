"""Rotary positions, the 16-bit cache and verified drafts: what the Python entry points refuse, and calls at the edge of what they take."""
import pytest
import torch

from test_gpu_kv16 import Setup, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu


def leaf(t):
    return t.clone().requires_grad_()


def refused(pv, what, calls):  # noqa: F811
    for i, call in enumerate(calls):
        with pytest.raises(pv.PVError, match=what):
            call()
            pytest.fail(f"call {i} went through")


@pytest.fixture
def at(pv):  # noqa: F811
    s = Setup(pv, [20], [3], heads=2, hd=64)
    s.fill_prefix()
    s.k, s.v, s.q = s.draw(3).cuda(), s.draw(3).cuda(), torch.randn(3, 4, 64, device="cuda").bfloat16()
    s.rot = pv.Rotary(64)
    s.pool.append(s.seqs(), s.k, s.v)
    s.x, s.u, s.tokens, s.begin = torch.randn(3, 100, device="cuda"), torch.rand(3, 2, device="cuda"), dev([1, 2, 3]), dev([0, 3])
    s.before = torch.nan_to_num(s.pool.pages)
    return s


def test_tensors_that_require_gradients(pv, at):  # noqa: F811
    s, p = at, dev([0, 1, 2])
    q = torch.softmax(s.x, 1)
    refused(pv, "gradient", [
        lambda: s.pool.append(s.seqs(), leaf(s.k), s.v), lambda: s.pool.append(s.seqs(), s.k, leaf(s.v)), lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=s.rot, q=leaf(s.q)),
        lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=s.rot, q=s.q, q_out=leaf(s.q)), lambda: s.rot.rotate(leaf(s.q), p), lambda: s.rot.rotate(s.q, p, out=leaf(s.q)),
        lambda: s.pool.attention(s.seqs(), leaf(s.q)), lambda: s.pool.attention(s.seqs(), leaf(s.q) * 1), lambda: s.pool.attention(s.seqs(), s.q, out=leaf(s.q)),
        lambda: s.pool.attention(s.seqs(), s.q, lse=torch.zeros(3, 4, device="cuda", requires_grad=True)), lambda: s.pool.attention(s.seqs(), leaf(s.q), stream=torch.cuda.Stream()),
        lambda: pv.verify_drafts(s.begin, leaf(s.x), s.tokens, s.u), lambda: pv.verify_drafts(s.begin, s.x, s.tokens, leaf(s.u)), lambda: pv.verify_drafts(s.begin, s.x, s.tokens, s.u, draft_probs=leaf(q)),
        lambda: pv.verify_drafts(s.begin, s.x, s.tokens, s.u, temperature=torch.ones(1, device="cuda", requires_grad=True)),
        lambda: pv.KV16Pool(4, 2, 64, pages=torch.zeros(4, 2, 2, 1024, dtype=torch.bfloat16, device="cuda", requires_grad=True))])
    assert torch.equal(torch.nan_to_num(s.pool.pages), s.before)
    out, turned, verdict = s.pool.attention(s.seqs(), s.q), s.rot.rotate(s.q, p), pv.verify_drafts(s.begin, s.x, s.tokens, s.u)
    lk, lv, lq, lx = leaf(s.k), leaf(s.v), leaf(s.q), leaf(s.x)
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            s.pool.append(s.seqs(), lk, lv)
            assert torch.equal(torch.nan_to_num(s.pool.pages), s.before) and torch.equal(s.pool.attention(s.seqs(), lq), out) and torch.equal(s.rot.rotate(lq, p), turned)
            again = pv.verify_drafts(s.begin, lx, s.tokens, s.u)
            assert torch.equal(again.accepted, verdict.accepted) and torch.equal(again.next_token, verdict.next_token) and torch.equal(again.probs, verdict.probs)


def test_shapes_types_and_places(pv, at):  # noqa: F811
    s, p = at, dev([0, 1, 2])
    wide = torch.zeros(3, 4, 128, device="cuda", dtype=torch.bfloat16)
    for bad in (s.q.cpu(), s.q[0], s.q[..., :32], s.q.double(), wide[..., ::2], None, s.q.transpose(1, 2).contiguous()):
        refused(pv, "x|rows|features|tensor", [lambda: s.rot.rotate(bad, p)])
        refused(pv, "q", [lambda: s.pool.attention(s.seqs(), bad), lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=s.rot, q=bad if bad is not None else s.q[:2])])
        refused(pv, "out", [lambda: s.rot.rotate(s.q, p, out=bad if bad is not None else s.q[:2]), lambda: s.pool.attention(s.seqs(), s.q, out=bad if bad is not None else s.q[:2])])
    for bad in (s.k.cpu(), s.k[:, :1], s.k[..., :32], s.k.double(), s.k[:2], s.k.half()):
        refused(pv, "k|v", [lambda: s.pool.append(s.seqs(), bad, s.v), lambda: s.pool.append(s.seqs(), s.k, bad)])
    for bad in (p.cpu(), p.long(), p[:2], dev([0, 0, 1, 1, 2, 2])[::2], [0, 1, 2]):
        refused(pv, "positions", [lambda: s.rot.rotate(s.q, bad), lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=s.rot, positions=bad)])
    refused(pv, "rotary|queries", [lambda: s.pool.append(s.seqs(), s.k, s.v, q=s.q), lambda: s.pool.append(s.seqs(), s.k, s.v, positions=p), lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=pv.Rotary(128)),
                                   lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=1)])
    refused(pv, "q_out", [lambda: s.pool.append(s.seqs(), s.k, s.v, rotary=s.rot, q_out=s.q)])
    refused(pv, "seqs", [lambda: s.pool.append(None, s.k, s.v), lambda: s.pool.attention((0, 1), s.q), lambda: s.pool.keep(None, p, dev([0]))])
    refused(pv, "type|dtype|of", [lambda: s.pool.attention(s.seqs(), s.q.half()), lambda: s.pool.attention(s.seqs(), s.q.float())])
    refused(pv, "n_q_heads", [lambda: s.pool.attention(s.seqs(), s.q[:, :3])])
    refused(pv, "scale", [lambda: s.pool.attention(s.seqs(), s.q, scale=float("nan")), lambda: s.pool.attention(s.seqs(), s.q, scale=float("inf"))])
    m = dev([1, 2, 3], torch.int64)
    refused(pv, "mask", [lambda: s.pool.attention(s.seqs(), s.q, mask=x) for x in (m.cpu(), m[:2], m.int(), m.view(3, 1, 1), m.view(3, 1)[:, :0], m.repeat(2)[::2], [1, 2, 3])])
    refused(pv, "lse", [lambda: s.pool.attention(s.seqs(), s.q, lse=torch.zeros(x, device="cuda", dtype=t)) for x, t in (((3, 3), torch.float32), ((4, 3), torch.float32), ((3, 4), torch.float64))])
    refused(pv, "path", [lambda: s.pool.keep(s.seqs(), x, dev([0])) for x in (p.cpu(), p.long(), p.view(1, 3), p.repeat(2)[::2])])
    refused(pv, "accepted", [lambda: s.pool.keep(s.seqs(), p, x) for x in (dev([0, 1]), dev([0]).cpu(), dev([0]).long(), 0)])
    refused(pv, "16|multiple|align|stride", [lambda: s.rot.rotate(torch.zeros(3 * 4 * 64 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(3, 4, 64), p),
                                             lambda: s.pool.attention(s.seqs(), torch.zeros(3, 4 * 64 + 4, device="cuda", dtype=torch.bfloat16)[:, :256].view(3, 4, 64))])
    assert torch.equal(torch.nan_to_num(s.pool.pages), s.before)


def test_verification_shapes_types_and_places(pv, at):  # noqa: F811
    s, call = at, pv.verify_drafts
    good = torch.softmax(s.x, 1)
    refused(pv, "logits", [lambda: call(s.begin, x, s.tokens, s.u) for x in (s.x.cpu(), s.x[0], s.x.double(), s.x.repeat(1, 2)[:, ::2])])
    refused(pv, "row_start", [lambda: call(x, s.x, s.tokens, s.u) for x in (s.begin.cpu(), s.begin.long(), s.begin.view(1, 2), s.begin[:0], [0, 3])])
    refused(pv, "tokens", [lambda: call(s.begin, s.x, x, s.u) for x in (s.tokens.cpu(), s.tokens.long(), s.tokens[:2])])
    refused(pv, "u must", [lambda: call(s.begin, s.x, s.tokens, x) for x in (s.u.cpu(), s.u.half(), s.u[:2], s.u.t().contiguous(), s.u.t().contiguous().t(), 0.5)])
    refused(pv, "draft_probs", [lambda: call(s.begin, s.x, s.tokens, s.u, draft_probs=x) for x in (good.cpu(), good.half(), good[:2], good[:, :99], good.repeat(1, 2)[:, ::2])])
    refused(pv, "parent", [lambda: call(s.begin, s.x, s.tokens, s.u, parent=x) for x in (s.tokens.cpu(), s.tokens.long(), s.tokens[:2])])
    refused(pv, "tree", [lambda: call(s.begin, s.x, s.tokens, s.u, draft_probs=good, parent=s.tokens)])
    refused(pv, "temperature", [lambda: call(s.begin, s.x, s.tokens, s.u, temperature=x) for x in (-1.0, float("nan"), torch.ones(2, device="cuda"), torch.ones(1), torch.ones(1, device="cuda").double())])
    refused(pv, "vocab", [lambda: call(s.begin, s.x[:, :0], s.tokens, s.u)])


def test_empty_calls(pv, at):  # noqa: F811
    s = at
    none = pv.KVSeqs(dev([0]), dev([]), torch.zeros(0, 4, dtype=torch.int32, device="cuda"))
    s.pool.append(none, s.k, s.v)
    assert torch.equal(torch.nan_to_num(s.pool.pages), s.before)
    out, lse = torch.full_like(s.q, 7.0), torch.full((3, 4), 7.0, device="cuda")
    s.pool.attention(none, s.q, out=out, lse=lse)
    assert (out == 7).all() and (lse == 7).all()
    empty = s.seqs(start=[0, 0])
    assert s.pool.attention(empty, s.q[:0]).shape == (0, 4, 64) and s.rot.rotate(s.q[:0], dev([])).shape == (0, 4, 64) and s.rot.rotate(s.q[:, :0], dev([0, 1, 2])).shape == (3, 0, 64)
    s.pool.append(empty, s.k[:0], s.v[:0])
    s.pool.keep(empty, dev([]), dev([0]))
    s.pool.keep(none, dev([0, 1, 2]), dev([]))
    assert torch.equal(torch.nan_to_num(s.pool.pages), s.before)
    got = pv.verify_drafts(dev([0]), s.x[:0], dev([]), s.u[:0])
    assert got.accepted.numel() == got.next_token.numel() == got.probs.numel() == 0
    got = pv.verify_drafts(dev([0, 0, 0]), s.x[:0], dev([]), s.u[:0], parent=dev([]))
    assert got.accepted.tolist() == [0, 0] and got.next_token.tolist() == [-1, -1]


def test_one_row_for_all_and_pages_shared_by_sequences(pv, at):  # noqa: F811
    """Inputs that are expanded; sequences whose prefixes are the same pages."""
    s = at
    one = s.k[:1]
    s.pool.append(s.seqs(), one.expand(3, 2, 64), one[:, :1].expand(3, 2, 64))
    a = torch.nan_to_num(s.pool.pages)
    s.pool.append(s.seqs(), one.repeat(3, 1, 1), one[:, :1].repeat(3, 2, 1))
    assert torch.equal(torch.nan_to_num(s.pool.pages), a)
    q = s.q[:1].expand(3, 4, 64)
    assert torch.equal(s.pool.attention(s.seqs(), q), s.pool.attention(s.seqs(), q.contiguous())) and torch.equal(s.rot.rotate(q, dev([5, 6, 7])), s.rot.rotate(q.contiguous(), dev([5, 6, 7])))
    x = s.x[:1].expand(3, 100)
    got, want = pv.verify_drafts(s.begin, x, s.tokens, s.u), pv.verify_drafts(s.begin, x.contiguous(), s.tokens, s.u)
    assert torch.equal(got.accepted, want.accepted) and torch.equal(got.next_token, want.next_token) and torch.equal(got.probs, want.probs)
    twice = pv.KVSeqs(dev([0, 3, 6]), dev([20, 20]), dev(s.tables.repeat(2, axis=0)))
    out = s.pool.attention(twice, s.q.repeat(2, 1, 1))
    assert torch.equal(out[:3], out[3:]) and torch.equal(out[:3], s.pool.attention(s.seqs(), s.q))
