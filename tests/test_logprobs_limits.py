"""How many rows a call of pv_token_logprobs takes: what the header states, refused beforehand by the call that gives the workspace's size too (no GPU needed)."""
import ctypes

import pytest

from paper_2505_01572_amd import binding


def status(rows, vocab):
    L, need = binding.lib(), ctypes.c_size_t(12345)
    a = L.pv_token_logprobs_bytes(rows, vocab, 1, ctypes.byref(need))
    if a:
        # a refused call enqueues nothing, so it may be made here
        assert L.pv_token_logprobs(0x1000, vocab, 1, rows, vocab, 0x1000, 1, 0x1000, None, None, 1, 0x1000, 0x1000, 0x1000, 1 << 60, None) == a
    return a


@pytest.mark.parametrize("vocab,most", [(1, (1 << 24) - 1), (32, (1 << 24) - 1), (4096, (1 << 24) - 1), (4097, (1 << 22) - 1), (32768, (1 << 22) - 1), (32769, (1 << 21) - 1),
                                        (128256, (1 << 20) - 1), (1 << 21, (1 << 16) - 1)])
def test_rows_of_a_call(vocab, most):
    assert status(most, vocab) == 0 and status(1, vocab) == 0 and status(255, vocab) == 0
    assert status(most + 1, vocab) == -3 and status(1 << 24, vocab) == -3
    assert b"rows" in binding.lib().pv_last_error()
