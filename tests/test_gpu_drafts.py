"""Drafts verified by sampling against the definition in 64 bits (tests/kv16_ref.py).

Whole numbers have to be equal: both sides draw from sums of some 10^5 probabilities in 64 bits (off by less than 10^-11), and a random number falls that near to one of as many borders once in 10^6 draws.  probs, with a
drafter's probabilities: half a step of 32 bits, 2^-24 of the value, and 10^-11 of it.  Without: the row's sum has exponentials of 32 bits.  An exponent t (in powers of two) is off by 3 * 2^-24 |t| (the difference, the factor, their
product), which is less than 3 * 17 * ln 2 * 2^-24 of the sum where the mean |t| is the 17 of 2^17 equal tokens at most; the exponential by 2^-23, a sum of 32 numbers in one register by 32 * 2^-24: less than 2^-17 in all."""
import numpy as np
import pytest
import torch

import kv16_ref as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pv():
    assert torch.cuda.is_available()
    import paper_2505_01572_amd as pv
    return pv


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype).cuda()


class Step:
    """Ragged rows of logits, drafts near the target, random numbers."""

    def __init__(self, rows, vocab, dtype="f32", kind="drawn", temperature=None, seed=0, tail=0):
        r = self.r = np.random.default_rng(seed + vocab)
        self.kind, self.vocab = kind, vocab
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        n = self.n = int(self.start[-1]) + tail
        x = r.normal(size=(n, vocab)) * 2.5
        self.logits = torch.from_numpy(x).to(TYPES[dtype])
        near = x + r.normal(size=x.shape) * 0.7
        self.temperature = np.asarray([0.5 + 0.25 * (i % 4) for i in range(len(rows))] if temperature is None else temperature, dtype=np.float32)
        hot = np.concatenate([np.repeat(np.fmax(self.temperature, 0.3), rows), np.ones(tail)])
        e = np.exp((near - near.max(1, keepdims=True)) / hot[:, None])
        q = e / e.sum(1, keepdims=True)
        self.q = np.roll(q, 1, 0).astype(np.float32) if kind == "drawn" else None
        self.parent = None
        if kind == "tree":
            self.parent = np.concatenate([[-1] + [int(r.integers(max(0, (i - 1) // 3 - 1), (i - 1) // 3 + 1)) for i in range(1, m)] for m in rows if m] + [[-1] * tail]).astype(np.int32)
            self.tokens = np.zeros(n, np.int32)
            for s, m in enumerate(rows):
                for i in range(1, m):
                    over = self.start[s] + self.parent[self.start[s] + i]
                    self.tokens[self.start[s] + i] = np.argsort(-near[over])[r.integers(0, min(3, vocab))]      # (the same token under a node, too)
        else:
            above = np.roll(q, 1, 0)
            self.tokens = np.array([r.choice(vocab, p=a / a.sum()) if kind == "drawn" else np.argmax(a) for a in above], dtype=np.int32)
        self.u = r.random((n, 2)).astype(np.float32)

    def run(self, pv, u=None, logits=None, **kw):
        u = torch.from_numpy(self.u).cuda() if u is None else u
        return pv.verify_drafts(dev(self.start), self.logits.cuda() if logits is None else logits, dev(self.tokens), u, draft_probs=None if self.q is None else torch.from_numpy(self.q).cuda(),
                                parent=None if self.parent is None else dev(self.parent), temperature=torch.from_numpy(self.temperature).cuda(), **kw)

    def check(self, got, u=None):
        a, f, path, probs = ref.verify(self.start, self.logits.double().numpy(), self.tokens, self.u.astype(np.float64) if u is None else u, self.temperature.astype(np.float64), self.q, self.parent)
        assert got.accepted.cpu().tolist() == a.tolist()
        assert got.next_token.cpu().tolist() == f.tolist()
        if self.parent is None:
            assert got.path is None
        else:
            assert got.path.cpu().tolist() == path.tolist()
        gp = got.probs.double().cpu().numpy()
        off = 2.0 ** -24 + (1e-11 if self.q is not None else 2.0 ** -17)
        assert (np.abs(gp - probs) <= off * probs + 2.0 ** -149).all()
        return a


ROWS = [[1], [2], [9], [3, 1, 5], [2] * 70, [0, 4, 0, 1, 6], [40]]


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 50, 257, 4095, 4096, 4097, 4099, 9001])
@pytest.mark.parametrize("rows", ROWS, ids=lambda r: "-".join(map(str, r[:5])))
def test_verify(pv, rows, vocab, dtype, kind):
    if len(rows) > 10 and vocab > 5000:
        rows = rows[:10]
    s = Step(rows, vocab, dtype, kind, tail=2)
    s.check(s.run(pv))


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
def test_a_large_vocabulary(pv, kind):
    some = 0
    for seed in range(3):
        s = Step([6, 9, 4], 128256, "bf16" if seed else "f32", kind, seed=seed)
        some += s.check(s.run(pv)).sum()
    assert some > 0 or kind != "drawn"                                  # (one given token of 128256 is hardly ever taken)


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
def test_many_draws(pv, kind):
    """Each sequence another one: refusals at every place."""
    s = Step([5] * 200, 300, "f32", kind, seed=3)
    a = s.check(s.run(pv))
    assert {0, 1, 2}.issubset(set(a.tolist())) if kind != "given" else a.max() > 0


@pytest.mark.parametrize("kind", ["drawn", "given", "tree"])
def test_temperatures(pv, kind):
    """0, less, NaN: the most probable token; tiny, huge and infinite ones."""
    t = [0.0, -1.0, float("nan"), 1e-30, 1e-45, 0.01, 50.0, 1e30, float("inf"), 1.0]
    for seed in range(4):
        s = Step([4] * len(t), 1000, "f32", kind, temperature=t, seed=seed)
        s.check(s.run(pv))


def test_equal_logits_take_the_lowest_id(pv):
    for dtype in ("f32", "bf16"):
        s = Step([3, 3], 5000, dtype, "given", temperature=[0.0, 0.0])
        s.logits[:] = -1.0
        s.logits[:, [77, 4321]] = 2.0
        s.logits[3:, 12] = 2.0
        s.tokens[:] = [0, 77, 4321, 0, 12, 12]
        got = s.run(pv)
        s.check(got)
        assert got.accepted.tolist() == [1, 2] and got.next_token.tolist() == [77, 12]


def test_random_numbers_of_64_bits_and_at_their_ends(pv):
    for kind in ("drawn", "given", "tree"):
        s = Step([4] * 30, 500, "f32", kind, seed=8)
        u = s.r.random((s.n, 2))
        u[::5, 1], u[1::5, 1], u[2::7, 0], u[3::7, 0] = 0.0, 1 - 2.0 ** -53, 0.0, 1 - 2.0 ** -53
        s.check(s.run(pv, u=torch.from_numpy(u).cuda()), u)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_masked_logits(pv, dtype):
    """-infinity and NaN have no probability; rows of nothing else, and with +infinity, have none at all."""
    s = Step([5] * 8, 700, dtype, "given", seed=5)
    s.logits[:, 100:] = -float("inf")
    s.logits[3, 7] = float("nan")
    s.logits[6] = -float("inf")
    s.logits[10] = float("nan")
    s.logits[16, 3] = float("inf")
    s.logits[20:25, 1:] = -float("inf")                                   # one token alone
    s.tokens[20:25] = 0
    s.tokens[30], s.tokens[31], s.tokens[36] = -1, 700, 2 ** 31 - 1
    got = s.run(pv)
    s.check(got)
    assert got.next_token[2].item() == -1 and got.accepted[4].item() == 4 and got.next_token[4].item() == 0
    t = Step([5] * 8, 700, dtype, "tree", seed=6)
    t.logits[:, 3:] = -float("inf")                                       # three tokens, all of them drafted: nothing is left to draw
    t.tokens[:] = t.r.integers(0, 3, t.n)
    t.logits[5] = -float("inf")
    t.check(t.run(pv))


def test_drafter_that_is_the_target(pv):
    """p = q: everything is taken; a draft the drafter cannot have drawn (q = 0): taken where the target has it."""
    s = Step([6] * 10, 800, "f32", "drawn", temperature=[1.0] * 10)
    p = np.stack([ref.probabilities(x, 1.0) for x in s.logits.double().numpy()])
    s.q = np.roll(p, 1, 0).astype(np.float32)
    s.u[:, 0] = 1 - 2.0 ** -20
    got = s.run(pv)
    s.check(got)
    assert got.accepted.tolist() == [5] * 10
    s.q[:, :] = 0
    s.check(s.run(pv))
    s.q[2, 5], s.q[9, 4], s.q[14] = float("nan"), float("inf"), float("nan")
    s.check(s.run(pv))


def test_nothing_left_of_the_difference(pv):
    """q above p everywhere (it is not normalised): a refusal draws from p."""
    s = Step([2] * 20, 300, "f32", "drawn", temperature=[1.0] * 20)
    p = np.stack([ref.probabilities(x, 1.0) for x in s.logits.double().numpy()])
    s.q = np.roll(p * 1.5, 1, 0).astype(np.float32)
    s.u[:, 0] = 0.9
    got = s.run(pv)
    s.check(got)
    assert got.accepted.tolist() == [0] * 20


def test_siblings_of_one_token_and_parents_that_are_none(pv):
    s = Step([8, 8, 8], 60, "f32", "tree", temperature=[1.0] * 3)
    s.parent[:] = [-1, 0, 0, 0, 1, 1, 2, 3, 5, 0, 9, 3, 4, 2, 6, -7, 0, 0, 1, 1, 2, 2, 3, 2 ** 31 - 1]
    s.tokens[1:4] = 5
    s.tokens[17] = s.tokens[18] = int(s.logits[16].argmax())
    for k in range(20):
        s.u = s.r.random((s.n, 2)).astype(np.float32)
        s.check(s.run(pv))


def test_trees_of_more_nodes_than_are_looked_at_at_once(pv):
    s = Step([2500, 1100], 40, "f32", "tree", temperature=[1.0, 0.8], seed=2)
    s.parent[1:1200] = 0                                                  # one node with children on both sides of a border
    s.tokens[1:1200] = s.r.integers(0, 40, 1199)
    s.logits[0, :38] = -30.0
    s.tokens[1:1100] = s.r.integers(0, 38, 1099)
    s.tokens[1100:1200] = 38
    for k in range(4):
        s.u = s.r.random((s.n, 2)).astype(np.float32)
        s.u[1:1100, 0] = 0.999
        s.check(s.run(pv))


def test_rows_of_any_stride(pv):
    for dtype in ("bf16", "f16", "f32"):
        for pad in (1, 2, 3, 8):
            s = Step([4, 3], 4111, dtype, "drawn")
            wide = torch.full((s.n, 4111 + pad), 9.0, dtype=TYPES[dtype], device="cuda")
            wide[:, pad:] = s.logits.cuda()
            s.check(s.run(pv, logits=wide[:, pad:]))
    one = torch.randn(1, 900, device="cuda").expand(5, 900)               # one row for all
    s = Step([5], 900, "f32", "given")
    s.logits = one.cpu().contiguous()
    s.check(s.run(pv, logits=one))


def test_a_number_for_the_temperature_and_empty_calls(pv):
    s = Step([4, 4], 100, "f32", "given", temperature=[0.7, 0.7])
    args = (dev(s.start), s.logits.cuda(), dev(s.tokens), torch.from_numpy(s.u).cuda())
    s.check(pv.verify_drafts(*args, temperature=float(np.float32(0.7))))
    z = pv.verify_drafts(dev([0, 0, 0]), s.logits[:0].cuda(), dev([]), torch.zeros(0, 2, device="cuda"))
    assert z.accepted.tolist() == [0, 0] and z.next_token.tolist() == [-1, -1] and z.probs.shape == (0,)
    z = pv.verify_drafts(dev([0]), s.logits.cuda(), dev(s.tokens), args[3])
    assert z.accepted.shape == (0,)


def test_captured_twice_with_work_between(pv):
    """Two graphs at a time, replayed in turn, data changed in place."""
    steps = [Step([5, 3, 9], 5000, "f32", k, seed=9) for k in ("drawn", "tree")]
    held, graphs, outs = [], [], []
    for s in steps:
        t = dict(start=dev(s.start), logits=s.logits.cuda(), tokens=dev(s.tokens), u=torch.from_numpy(s.u).cuda(), q=None if s.q is None else torch.from_numpy(s.q).cuda(),
                 parent=None if s.parent is None else dev(s.parent), temperature=torch.from_numpy(s.temperature).cuda())

        def call(t=t):
            return pv.verify_drafts(t["start"], t["logits"], t["tokens"], t["u"], draft_probs=t["q"], parent=t["parent"], temperature=t["temperature"])
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        held.append((t, call)); graphs.append(g)
    for i in range(4):
        for s, (t, call), g, out in zip(steps, held, graphs, outs):
            s.u = s.r.random((s.n, 2)).astype(np.float32)
            t["u"].copy_(torch.from_numpy(s.u))
        for g in graphs:
            g.replay()
        for s, (t, call), out in zip(steps, held, outs):
            s.check(out)
            s.check(call())


def test_two_calls_at_once(pv):
    """On two streams; the inputs stay alive until both have run."""
    steps = [Step([7, 2, 5], 30000, "f32", "drawn", seed=1), Step([30, 2], 30000, "bf16", "tree", seed=2)]
    held = [dict(row_start=dev(s.start), logits=s.logits.cuda(), tokens=dev(s.tokens), u=torch.from_numpy(s.u).cuda(), draft_probs=None if s.q is None else torch.from_numpy(s.q).cuda(),
                 parent=None if s.parent is None else dev(s.parent), temperature=torch.from_numpy(s.temperature).cuda()) for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = [[pv.verify_drafts(**h, stream=x) for h, x in zip(held, streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for s, g in zip(steps, pair):
            s.check(g)


def test_frequencies_are_the_targets(pv):
    """Tokens behind a draft come out as the target alone would draw them: 200000 sequences of two rows over eight tokens, each frequency within five standard deviations."""
    n, v = 200000, 8
    g = torch.Generator(device="cuda"); g.manual_seed(1)
    row = torch.randn(v, generator=g, device="cuda")
    p, q = torch.softmax(row.double(), 0), torch.softmax(torch.randn(v, generator=g, device="cuda"), 0)
    start = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    tokens = torch.multinomial(q, 2 * n, replacement=True, generator=g).to(torch.int32)
    u = torch.rand(2 * n, 2, generator=g, device="cuda", dtype=torch.float64)
    for kw in (dict(draft_probs=q.expand(2 * n, v)), dict(), dict(parent=torch.tensor([-1, 0], dtype=torch.int32, device="cuda").repeat(n))):
        got = pv.verify_drafts(start, row.expand(2 * n, v), tokens, u, **kw)
        first = torch.where(got.accepted == 1, tokens[1::2], got.next_token).long()
        seen = torch.bincount(first, minlength=v).double() / n
        assert ((seen - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()
