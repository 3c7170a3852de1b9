"""Trees whose nodes' children hold all that a row allows: one of them is taken whatever the random numbers, and a token follows.

What is left behind refused children is what the remaining tokens weigh, not 1 less a rounded sum.  Against the definition in 64 bits (tests/kv16_ref.py), whole numbers equal: weights are off by some 10^-12 of themselves, and the
comparisons u * (what is left) < p of these cases lie further from equality than that."""
import numpy as np
import pytest
import torch

import kv16_ref as ref
from test_gpu_drafts import TYPES, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu

ENDS = {"f32": (torch.float32, 1 - 2.0 ** -24), "f64": (torch.float64, 1 - 2.0 ** -53)}


def same(got, a, f, path):
    for name, have, want in (("accepted", got.accepted, a), ("path", got.path, path), ("next_token", got.next_token, f)):
        other = np.nonzero(have.cpu().numpy() != want)[0]
        assert len(other) == 0, (name, len(other), other[:8], have.cpu().numpy()[other[:8]], want[other[:8]])


def verdict(pv, start, logits, tokens, parent, u, t):  # noqa: F811
    got = pv.verify_drafts(dev(start), logits.cuda(), dev(tokens), u.cuda(), parent=dev(parent), temperature=torch.full((len(start) - 1,), t, dtype=torch.float32, device="cuda"))
    a, f, path, _ = ref.verify(start, logits.double().numpy(), tokens, u.double().numpy(), [float(np.float32(t))] * (len(start) - 1), None, parent)
    same(got, a, f, path)
    return got


def allowed(n, ids, apart, vocab, dtype, seed):
    """Rows in groups of 1 + len(ids): a root that allows `ids` alone, `apart` [n, len(ids)] below the first, and children that allow three tokens."""
    r, m = np.random.default_rng(seed), 1 + len(ids)
    x = np.full((n, m, vocab), -np.inf)
    x[:, 0, ids] = 3.0 - apart
    x[:, 1:, [0, vocab // 3, vocab - 1]] = r.normal(size=(n, m - 1, 3))
    return torch.from_numpy(x.reshape(n * m, vocab)).to(TYPES[dtype])


@pytest.mark.parametrize("order", ["first", "last"])
@pytest.mark.parametrize("bits", list(ENDS))
@pytest.mark.parametrize("dtype,t", [("f32", 1.0), ("f32", 0.3), ("bf16", 1.0), ("f16", 2.5)])
def test_two_tokens_both_drafted(pv, dtype, t, bits, order):  # noqa: F811
    """Differences from 0 to 16, the more probable one tried first or last, u at its upper end, at 0, and drawn."""
    n, vocab = 1023, 40
    ids = [7, 31] if order == "first" else [31, 7]
    apart = np.zeros((n, 2))
    apart[:, 1] = np.arange(n) / 64.0
    logits = allowed(n, [7, 31], apart, vocab, dtype, 1)
    start = np.arange(0, 3 * n + 1, 3)
    tokens, parent = np.tile([0, *ids], n).astype(np.int32), np.tile([-1, 0, 0], n).astype(np.int32)
    kind, end = ENDS[bits]
    for first in (end, 0.0, None):
        u = torch.rand(3 * n, 2, dtype=kind, generator=torch.Generator().manual_seed(5))
        if first is not None:
            u[:, 0] = first
        got = verdict(pv, start, logits, tokens, parent, u, t)
        assert bool((got.accepted == 1).all()) and bool((got.next_token >= 0).all())


@pytest.mark.parametrize("bits", list(ENDS))
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [3, 4097, 30001])
def test_three_tokens_all_drafted(pv, vocab, dtype, bits):  # noqa: F811
    """In different segments of a row, tried in any order, one of them twice; ids that are none between them."""
    r = np.random.default_rng(vocab)
    n = 200 if vocab < 30000 else 40
    ids = [0, vocab // 2, vocab - 1]
    apart = r.integers(0, 10 * 64, (n, 3)) / 64.0
    x = torch.full((6 * n, vocab), -float("inf"))
    x[::6, ids] = torch.from_numpy(3.0 - apart).float()
    for i in range(1, 6):
        x[i::6, ids] = torch.from_numpy(r.normal(size=(n, 3))).float()
    logits = x.to(TYPES[dtype])
    tokens = np.zeros((n, 6), np.int32)
    for s in range(n):
        order = r.permutation(ids)
        tokens[s, 1:] = [order[0], order[0] if s % 2 else -1, order[1], vocab if s % 3 else order[1], order[2]]
    parent = np.tile([-1, 0, 0, 0, 0, 0], n).astype(np.int32)
    kind, end = ENDS[bits]
    for first in (end, 0.0, None):
        u = torch.rand(6 * n, 2, dtype=kind, generator=torch.Generator().manual_seed(6))
        if first is not None:
            u[:, 0] = first
        got = verdict(pv, np.arange(0, 6 * n + 1, 6), logits, tokens.reshape(-1), parent, u, 1.0)
        assert bool((got.accepted == 1).all()) and bool((got.next_token >= 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_tokens_of_a_row_drafted(pv, dtype):  # noqa: F811
    """Some thousand children on both sides of what is looked at at once; levels below; a row that begins between four bytes."""
    r, vocab = np.random.default_rng(3), 1501
    order, m = r.permutation(vocab), 1 + vocab + 4
    x = np.full((m, vocab), -np.inf)
    x[0] = np.where(np.arange(vocab) % 3 == 0, r.normal(size=vocab) * 3, -np.inf)
    x[1:, [2, 9]] = [1.0, -4.0]
    wide = torch.zeros(m, vocab + 1)
    wide[:, 1:] = torch.from_numpy(x).float()
    logits = wide.to(TYPES[dtype])
    last = 1 + int(np.nonzero(order % 3 == 0)[0][-1])                     # the last child that the row allows
    tokens = np.concatenate([[0], order, [9, 2, 2, 9]]).astype(np.int32)
    parent = np.concatenate([[-1], np.zeros(vocab), [last, last, m - 3, m - 3]]).astype(np.int32)
    for kind, end in ENDS.values():
        u = torch.full((m, 2), end, dtype=kind)
        rows = logits[:, 1:]
        dl = logits.cuda()[:, 1:]
        got = pv.verify_drafts(dev([0, m]), dl, dev(tokens), u.cuda(), parent=dev(parent), temperature=1.0)
        a, f, path, _ = ref.verify(np.array([0, m]), rows.double().numpy(), tokens, u.double().numpy(), [1.0], None, parent)
        same(got, a, f, path)
        assert a[0] >= 1 and f[0] >= 0
