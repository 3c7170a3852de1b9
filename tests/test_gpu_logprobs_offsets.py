"""Log probabilities of rows whose logits all lie far from zero, against 64 bits.

log p = (x - M) - ln Z has no term of the size of the logits: x - M is off by 2^-24 of itself, Z by less than 2^-17 of itself (tests/test_gpu_logprobs.py).  So 2^-17 + 2^-22 |log p|, whatever the offset;
entropy as there; lse = M + ln Z is rounded once more, 2^-24 of itself."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import TYPES, oracle, pv  # noqa: F401

pytestmark = pytest.mark.gpu


def check(got, x, tokens, top):
    want = oracle(x.double().cpu().numpy(), tokens.cpu().numpy(), top)
    assert np.array_equal(got.top_ids.cpu().numpy(), want["top_ids"])
    for name in ("logprobs", "top_logprobs"):
        g, w = getattr(got, name).double().cpu().numpy(), want[name]
        assert np.isfinite(g).all()
        assert (np.abs(g - w) <= 2.0 ** -17 + 2.0 ** -22 * np.abs(w)).all(), (name, np.abs(g - w).max())
    e, l = got.entropy.double().cpu().numpy(), got.lse.double().cpu().numpy()
    assert (np.abs(e - want["entropy"]) <= 2.0 ** -16 * (1 + want["entropy"] + np.log(x.shape[1]))).all(), np.abs(e - want["entropy"]).max()
    assert (np.abs(l - want["lse"]) <= 2.0 ** -17 + 2.0 ** -23 * np.abs(want["lse"])).all()


@pytest.mark.parametrize("rows,vocab", [(3, 50), (5, 4097), (4, 32000), (3, 128256), (260, 33001)])
@pytest.mark.parametrize("offset", [1e3, -1e3, 1e5, -3e5, 1e7, -1.1e7, 2e10, -7e12, 1e30, -3e38])
def test_common_offsets(pv, rows, vocab, offset):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    x[rows // 2] *= max(1.0, abs(offset) * 2.0 ** -22)               # (and a row that is not flat where steps are large)
    x = x + offset
    tokens = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda", dtype=torch.int32)
    check(pv.token_logprobs(x, tokens, top=9), x, tokens, 9)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("offset", [300.0, -300.0, 5000.0, -60000.0])
def test_common_offsets_in_16_bits(pv, dtype, offset):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(9)
    for vocab in (700, 40000):
        x = (torch.randn(4, vocab, generator=g, device="cuda") * 3 + offset).to(TYPES[dtype])
        tokens = torch.randint(0, vocab, (4, 2), generator=g, device="cuda", dtype=torch.int32)
        check(pv.token_logprobs(x, tokens, top=9), x, tokens, 9)


def test_every_thread_with_a_maximum_of_its_own(pv):  # noqa: F811
    """Logits from -5e8 to 5e8 beside each other: threads whose largest logit is near and far from zero are joined."""
    g = torch.Generator(device="cuda").manual_seed(10)
    for vocab in (300, 32768, 128256):
        x = (torch.rand(6, vocab, generator=g, device="cuda") - 0.5) * torch.tensor([1e3, 1e5, 1e7, 1e9, 3e2, 3e4], device="cuda").view(6, 1)
        x[3:] = x[3:].sort(1).values
        tokens = torch.randint(0, vocab, (6, 5), generator=g, device="cuda", dtype=torch.int32)
        check(pv.token_logprobs(x, tokens, top=9), x, tokens, 9)
