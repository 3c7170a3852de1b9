"""Log probabilities, entropy and alternatives against 64 bits.

In 32 bits: x - M and its product with log2(e) are off by 2^-24 of it each and the exponential by 2^-22, in sums whose terms are added over 32 numbers, 64 lanes, 16 waves and 64 segments (chains of under 64
additions): Z and the entropy's sum are off by less than 2^-17 of themselves for logits less than 88 below the maximum (further ones add nothing).  So log probabilities: 2^-17 + 2^-22 of |logit| and |lse|;
entropy: 2^-16 (1 + H + log Z)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pv():
    assert torch.cuda.is_available()
    import paper_2505_01572_amd as pv
    return pv


def oracle(x, tokens, top):
    """numpy, 64 bits, a row at a time: NaN as -infinity, ties to the lower id."""
    rows = x.shape[0]
    out = dict(logprobs=np.full(tokens.shape, np.nan), entropy=np.zeros(rows), lse=np.zeros(rows), top_ids=np.zeros((rows, top), np.int64), top_logprobs=np.zeros((rows, top)))
    for r in range(rows):
        v = np.where(np.isnan(x[r]), -np.inf, x[r])
        order = np.argsort(-v, kind="stable")[:top]
        out["top_ids"][r] = order
        m = v.max()
        if m == -np.inf:
            out["lse"][r] = -np.inf
            lp = np.full(v.shape, -np.inf)
        elif m == np.inf:
            out["lse"][r], out["entropy"][r], lp = np.nan, np.nan, np.full(v.shape, np.nan)
        else:
            z = np.exp(v - m).sum()
            out["lse"][r] = m + np.log(z)
            lp = (v - m) - np.log(z)
            p = np.exp(lp)
            out["entropy"][r] = -(p[p > 0] * lp[p > 0]).sum()
        out["top_logprobs"][r] = lp[order]
        ok = (tokens[r] >= 0) & (tokens[r] < len(v))
        out["logprobs"][r, ok] = lp[tokens[r, ok]]
    return out


def check(got, x, tokens, top):
    want = oracle(x.double().cpu().numpy(), tokens.cpu().numpy(), top)
    assert np.array_equal(got.top_ids.cpu().numpy(), want["top_ids"])

    def near(g, w, slack):
        g = g.double().cpu().numpy()
        assert np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(np.isneginf(g), np.isneginf(w))
        f = np.isfinite(w)
        assert (np.abs(g - w)[f] <= np.broadcast_to(slack, w.shape)[f]).all(), np.abs(g - w)[f].max()
    with np.errstate(invalid="ignore"):
        lse = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0.0)
        near(got.lse, want["lse"], 2.0 ** -17 + 2.0 ** -22 * lse)
        for name in ("logprobs", "top_logprobs"):
            near(getattr(got, name), want[name], 2.0 ** -17 + 2.0 ** -22 * (np.abs(np.where(np.isfinite(want[name]), want[name], 0)) + 2 * lse[:, None]))
        near(got.entropy, want["entropy"], 2.0 ** -16 * (1 + want["entropy"] + np.log(x.shape[1])))


CASES = [(1, 1, 1, 1), (3, 2, 1, 2), (5, 63, 3, 32), (2, 64, 1, 5), (7, 301, 1, 20), (4, 4096, 1, 32), (4, 4097, 2, 1), (2, 32000, 1, 20), (8, 128256, 1, 5), (1, 200003, 40, 32),
         (300, 5000, 1, 20), (257, 32768, 1, 3), (260, 33001, 0, 8), (2, 262145, 1, 7), (300, 64, 1, 0), (1, 2097152, 1, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,n,top", CASES)
def test_against_64_bits(pv, rows, vocab, n, top, dtype):
    g = torch.Generator(device="cuda").manual_seed(vocab + rows)
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(TYPES[dtype])
    tokens = torch.randint(0, vocab, (rows, n), generator=g, device="cuda", dtype=torch.int32)
    check(pv.token_logprobs(x, tokens, top=top), x, tokens, top)


@pytest.mark.parametrize("vocab", [100, 5000, 40000])
@pytest.mark.parametrize("rows", [12, 268])
def test_masks_ties_and_numbers_that_are_none(pv, rows, vocab):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    inf = float("inf")
    x[0] = 1.5                                     # all equal
    x[1] = -inf                                    # nothing left
    x[2, 7:] = -inf                                # seven tokens allowed
    x[3] = torch.finfo(torch.float32).min          # a mask of the type's lowest value, and two tokens
    x[3, 90], x[3, 3] = 2.0, 1.0
    x[4, ::3] = float("nan")
    x[5] = float("nan")
    x[6, 50] = inf
    x[7] = torch.floor(x[7])                       # many ties
    x[8, 11] = 3e38
    x[9] = torch.where(x[9] > 0, 0.0, -0.0)        # zeros of both signs are one number
    x[10] = 20.0
    x[10, 99] = 1e4
    x[11] = torch.finfo(torch.float32).min
    tokens = torch.tensor([0, vocab - 1, -1, vocab, 2 ** 31 - 1, 50, 3], dtype=torch.int32, device="cuda").repeat(rows, 1)
    check(pv.token_logprobs(x, tokens, top=20), x, tokens, 20)


def test_strided_rows_and_offsets(pv):
    """Rows of a wider array, addresses of every alignment."""
    g = torch.Generator(device="cuda").manual_seed(6)
    for t in TYPES.values():
        wide = (torch.randn(9, 5003, generator=g, device="cuda") * 3).to(t)
        for at in range(5):
            x = wide[:, at:at + 4500]
            tokens = torch.randint(0, 4500, (9,), generator=g, device="cuda", dtype=torch.int32)
            got = pv.token_logprobs(x, tokens, top=4)
            assert got.logprobs.shape == (9,)
            check(got._replace(logprobs=got.logprobs[:, None]), x, tokens[:, None], 4)
        one = wide[0:1, :700].expand(6, 700)        # the same row six times
        check(pv.token_logprobs(one, None, top=3), one, torch.zeros(6, 0, dtype=torch.int32), 3)


def test_runs_are_the_same_and_graphs_replay(pv):
    g = torch.Generator(device="cuda").manual_seed(7)
    x, tokens = torch.randn(16, 50000, generator=g, device="cuda"), torch.randint(0, 50000, (16, 2), generator=g, device="cuda", dtype=torch.int32)
    pv.token_logprobs(x, tokens, top=10)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pv.token_logprobs(x, tokens, top=10)
    for i in range(5):
        x.normal_(generator=g)
        x[3].round_()
        graph.replay()
        torch.cuda.synchronize()
        want = pv.token_logprobs(x, tokens, top=10)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    torch.cuda.synchronize()


def test_two_streams_at_once(pv):
    x, y = torch.randn(8, 128256, device="cuda"), torch.randn(300, 32000, device="cuda").to(torch.bfloat16)
    a, b = torch.arange(8, dtype=torch.int32, device="cuda"), torch.arange(600, dtype=torch.int32, device="cuda").view(300, 2)
    want = [pv.token_logprobs(x, a, top=5), pv.token_logprobs(y, b, top=20)]
    streams = [torch.cuda.Stream() for _ in want]
    for _ in range(4):
        got = []
        for s, args in zip(streams, ((x, a, 5), (y, b, 20))):
            s.wait_stream(torch.cuda.current_stream())
            got.append(pv.token_logprobs(*args, stream=s))
        torch.cuda.synchronize()
        for u, w in zip(got, want):
            assert all(torch.equal(i, j) for i, j in zip(u, w))
