"""Verified drafts over more than 64 segments of 4096 tokens a row, and in calls so large that a workgroup takes 8192 logits of a row, or 14336 (more than 4096 segments in all).  Oracle and tolerances: tests/test_gpu_drafts.py.

Odd vocabularies: rows of 16-bit numbers begin at any multiple of two bytes in turn."""
import numpy as np
import pytest
import torch

from test_gpu_drafts import Step, pv  # noqa: F401

pytestmark = pytest.mark.gpu

SOME, MOST = 300001, (1 << 21) - 1                                        # 74 and 512 segments


def step(vocab, dtype, kind, temperature, seed=0):
    return Step([4, 1, 5], vocab, dtype, kind, temperature=temperature, seed=seed, tail=1)


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [262144, 262145, SOME, MOST])
def test_verify(pv, vocab, dtype, kind):  # noqa: F811
    s = step(vocab, dtype, kind, [1.0, 0.7, 0.3], seed=1)
    s.check(s.run(pv))


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [SOME, MOST])
def test_most_probable_tokens(pv, vocab, dtype, kind):  # noqa: F811
    """T = 0: the lowest id of equal ones, in the first segments, beyond the 64th, the last token of all; a draft that is it."""
    s = step(vocab, dtype, kind, [0.0, 0.0, 0.0])
    s.logits.clamp_(max=8.0)
    for row, ids in enumerate([[0, vocab - 1], [vocab - 1], [262143, 262144], [299999, 300000], [5, 270000], [266241, 280000], [1], [4095, 4096], [vocab - 2], [123456]]):
        s.logits[row, ids] = 9.0
        if row + 1 < s.n and (s.parent is None or row < 3):
            s.tokens[row + 1] = ids[0]
    s.check(s.run(pv))


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [SOME, MOST])
def test_masked_logits(pv, vocab, dtype, kind):  # noqa: F811
    """Whole segments of -infinity or NaN; all that is probable beyond the 64th segment, or in one token; a row of nothing else; one with +infinity."""
    s = step(vocab, dtype, kind, [1.0, 0.8, 1.3], seed=2)
    x = s.logits
    x[0, :265000] = -np.inf
    x[1, ::3] = np.nan
    x[2, 4096:290000] = np.nan
    x[4, :] = -np.inf
    x[4, vocab - 1] = 1.0
    x[6, : vocab - 7] = -np.inf
    x[8, :] = np.nan
    x[9, 270001] = np.inf
    for k in range(3):
        s.u = s.r.random((s.n, 2)).astype(np.float32)
        got = s.run(pv)
        s.check(got)
        assert got.next_token[1].item() == vocab - 1
    s.u[:, 1] = 0.0                                                       # the first token that has any
    s.check(s.run(pv))


@pytest.mark.parametrize("vocab", [SOME, MOST])
def test_refused_tokens_take_their_part_with_them(pv, vocab):  # noqa: F811
    """Children of the first node that hold nearly all of p, in segments far apart, all refused: the draw is from what is left."""
    s = Step([6, 6], vocab, "bf16", "tree", temperature=[1.0, 1.0])
    ids = [0, 4096, 262144, 280000, vocab - 1]
    for first in (0, 6):
        s.parent[first + 1:first + 6] = 0
        s.tokens[first + 1:first + 6] = ids
        s.logits[first, ids] = 12.0
    for k in range(4):
        s.u = s.r.random((s.n, 2)).astype(np.float32)
        s.u[:, 0] = 1 - 2.0 ** -24
        got = s.run(pv)
        a = s.check(got)
        assert a.tolist() == [0, 0] and not set(got.next_token.tolist()) & set(ids)
