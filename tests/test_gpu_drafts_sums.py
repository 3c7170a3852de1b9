"""Verified drafts without a drafter's probabilities: what the exponentials of 32 bits leave of a row's sum.

A sum is made segment by segment, each relative to its own largest logit.  Of every 4096 tokens here one is some 9 powers of two above the others, which have eight ninths of the sum.  Their exponents are off by 2^-24 of 10
twice (the difference, its product with log2(e) / T), each on its own: over 10^6 tokens, with chances of less than 10^-9 otherwise, by 10 ln 2 * 2^-23 * sqrt(2 ln(2 10^9) / 10^6) < 2^-27 on average; sums of 16 to 28 numbers a
register, in thousands of threads, as little.  What all have in common counts whole: the exponential's own error, 2^-23 at most, and the rounding of p, 2^-24.  Together less than 2^-22 of p.  (A factor log2(e) / T in 32 bits, off by
2^-24 of itself at the temperatures here, would be off by 8/9 * 9 ln 2 * 2^-24 for all: 2^-21.5.)"""
import numpy as np
import pytest
import torch

import kv16_ref as ref
from test_gpu_drafts import TYPES, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu


def temperatures():
    """Of some thousand, those at which log2(e) / T is furthest, relative to itself, from a number of 32 bits: above and below it."""
    t = (0.72 + np.arange(8192) / 2.0 ** 17).astype(np.float32)
    c = np.log2(np.e) / t.astype(np.float64)
    off = c.astype(np.float32).astype(np.float64) / c - 1
    assert off.max() > 2.0 ** -24 * 0.9 and off.min() < -2.0 ** -24 * 0.9
    return [float(t[off.argmax()]), float(t[off.argmin()])]


@pytest.mark.parametrize("kind", ["given", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_what_all_tokens_have_in_common(pv, dtype, kind):  # noqa: F811
    vocab, r = 1 << 20, np.random.default_rng(4)
    for t in temperatures():
        x = r.uniform(-0.5, 0.5, vocab)
        x[777::4096] = 9.0 * np.log(2) * t
        logits = torch.from_numpy(np.tile(x, (2, 1))).to(TYPES[dtype])
        tokens, u = np.array([0, 777], np.int32), torch.zeros(2, 2)
        got = pv.verify_drafts(dev([0, 2]), logits.cuda(), dev(tokens), u.cuda(), parent=dev([-1, 0]) if kind == "tree" else None, temperature=t)
        p = ref.probabilities(logits[0].double().numpy(), float(np.float32(t)))[777]
        assert 0.0002 < p < 0.0008 and got.accepted.tolist() == [1]
        assert abs(got.probs[1].item() / p - 1) < 2.0 ** -22, (t, got.probs[1].item() / p - 1)


@pytest.mark.parametrize("kind", ["given", "tree"])
def test_masked_tokens_at_every_temperature(pv, kind):  # noqa: F811
    """-infinity has no weight, whichever way the factor is rounded."""
    x = torch.full((2, 9000), -float("inf"))
    x[:, [5, 4096, 8999]] = torch.tensor([1.0, 0.0, -1.0])
    for t in (*temperatures(), 1.0, 2.0 ** -100, 1e-45, 3e38, float("inf")):
        got = pv.verify_drafts(dev([0, 2]), x.cuda(), dev([0, 4096]), torch.full((2, 2), 0.25, device="cuda"), parent=dev([-1, 0]) if kind == "tree" else None, temperature=t)
        p = ref.probabilities(x[0].double().numpy(), float(np.float32(t)))[4096]
        assert abs(got.probs[1].item() - p) <= 2.0 ** -22 * p + 2.0 ** -126 and got.accepted.item() == int(p > 0.25)


@pytest.mark.parametrize("kind", ["given", "tree"])
def test_logits_and_temperatures_near_the_largest_number(pv, kind):  # noqa: F811
    """Factors of less than 2^-100, and such that are not normal (of 22 bits at T = 3e38: twice 2^-22 of an exponent of 1.5, and the rest as above: less than 2^-19)."""
    x = torch.full((2, 5000), -float("inf"))
    x[:, :5] = torch.tensor([1e38, 0.0, -2e38, 0.7e38, 0.99e38])
    x[:, 4100:4103] = torch.tensor([0.2e38, -1e38, 0.3e38])
    for t in (1e36, 1e37, 1e38, 3e38):
        got = pv.verify_drafts(dev([0, 2]), x.cuda(), dev([0, 4]), torch.full((2, 2), 0.01, device="cuda"), parent=dev([-1, 0]) if kind == "tree" else None, temperature=t)
        p = ref.probabilities(x[0].double().numpy(), float(np.float32(t)))[4]
        assert abs(got.probs[1].item() / p - 1) <= 2.0 ** -19 and got.accepted.item() == 1
