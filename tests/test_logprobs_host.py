"""What pv_token_logprobs refuses (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2505_01572_amd import binding, operators


def call(logits=0x1000, stride=64, dtype=0, rows=4, vocab=64, tokens=0x1000, n=1, logprobs=0x1000, top=2, ids=0x1000, tops=0x1000, ws=None, nbytes=0):
    return binding.lib().pv_token_logprobs(logits, stride, dtype, rows, vocab, tokens, n, logprobs, 0x1000, 0x1000, top, ids, tops, ws, nbytes, None)


def test_refusals():
    assert call(rows=-1) == call(rows=(1 << 24) + 1) == call(vocab=0) == call(vocab=(1 << 21) + 1) == call(top=-1) == call(top=33) == call(vocab=4, top=5) == call(n=-1) == -3
    assert call(dtype=3) == call(logits=None) == call(tokens=None) == call(logprobs=None) == call(ids=None) == call(tops=None) == call(stride=-1) == call(logits=0x1002) == call(logits=0x1001, dtype=1) == -1
    need = ctypes.c_size_t()
    assert binding.lib().pv_token_logprobs_bytes(4, 32768, 2, ctypes.byref(need)) == 0 and need.value == 0
    assert binding.lib().pv_token_logprobs_bytes(4, 40000, 2, ctypes.byref(need)) == 0 and need.value > 0
    assert call(vocab=40000, stride=40000) == call(vocab=40000, stride=40000, ws=0x1000, nbytes=need.value - 1) == -5
    assert call(vocab=40000, stride=40000, ws=0x1008, nbytes=need.value) == -1
    assert call(rows=1 << 24, vocab=32, stride=32) == -3          # more than a launch takes
    assert call(rows=0, logits=None) == 0


def test_cpu_tensors_are_refused():
    with pytest.raises(binding.PVError):
        operators.token_logprobs(torch.zeros(2, 8))
