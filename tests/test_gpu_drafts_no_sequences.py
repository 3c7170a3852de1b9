"""Rows of logits that belong to no sequence, because the call has none: probs 0 and path -1, as in rows behind the last sequence."""
import ctypes

import pytest
import torch

from test_gpu_drafts import dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("rows", [1, 3, 700])
def test_rows_without_sequences(pv, rows, tree):  # noqa: F811
    from paper_2505_01572_amd import binding
    L = binding.lib()
    x, tokens, u, up = torch.randn(rows, 50, device="cuda"), dev([0] * rows), torch.rand(rows, 2, device="cuda"), dev([-1] * rows)
    path, probs = torch.full((rows + 1,), 7, dtype=torch.int32, device="cuda"), torch.full((rows + 1,), 7.0, device="cuda")
    start, none = dev([0]), torch.full((4,), 7, dtype=torch.int32, device="cuda")
    b = ctypes.c_size_t()
    assert L.pv_verify_drafts_bytes(rows, 0, 50, ctypes.byref(b)) == 0 and b.value == 0
    for with_path in (True, False):
        if tree and not with_path:
            continue
        path.fill_(7), probs.fill_(7)
        rc = L.pv_verify_drafts(start.data_ptr(), 0, x.data_ptr(), 50, 0, rows, 50, tokens.data_ptr(), u.data_ptr(), 0, None, 0, up.data_ptr() if tree else None, None, 1.0, none.data_ptr(), none.data_ptr(),
                                path.data_ptr() if with_path else None, probs.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        assert bool((probs[:rows] == 0).all()) and bool((path[:rows] == (-1 if with_path else 7)).all()) and bool(probs[rows] == 7) and bool(path[rows] == 7) and bool((none == 7).all())
    got = pv.verify_drafts(start, x, tokens, u, parent=up if tree else None)
    assert bool((got.probs == 0).all()) and got.accepted.numel() == got.next_token.numel() == 0 and (bool((got.path == -1).all()) if tree else got.path is None)


def test_captured(pv):  # noqa: F811
    x, tokens, u, start = torch.randn(5, 50, device="cuda"), dev([0] * 5), torch.rand(5, 2, device="cuda"), dev([0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = pv.verify_drafts(start, x, tokens, u, parent=tokens)
    for _ in range(3):
        got.probs.fill_(7), got.path.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert bool((got.probs == 0).all()) and bool((got.path == -1).all())


def test_outputs_that_are_none(pv):  # noqa: F811
    """Refused where there are rows to write for."""
    from paper_2505_01572_amd import binding
    L = binding.lib()
    t = torch.zeros(64, dtype=torch.int32, device="cuda")
    call = lambda rows, parent, path, probs: L.pv_verify_drafts(t.data_ptr(), 0, t.data_ptr(), 2, 0, rows, 2, t.data_ptr(), t.data_ptr(), 0, None, 0, parent, None, 1.0, t.data_ptr(), t.data_ptr(), path, probs, None, 0, None)  # noqa: E731
    assert call(2, None, None, None) == -1 and call(2, t.data_ptr(), None, t.data_ptr()) == -1 and call(2, None, None, t.data_ptr() + 2) == -1
    assert call(0, None, None, None) == 0
