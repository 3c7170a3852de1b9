"""The operators of the 16-bit key/value cache against the 64-bit oracle (tests/kv16_ref.py).

Values, and keys that are not rotated, are rounded to the pool's type once: equal to torch's conversion, bit for bit, in the whole pool, and moved tokens likewise.  Rotated numbers: as in tests/test_gpu_rotary.py.
Attention: an output is off by half a step, eps / 2 of its value, plus what the arithmetic in 32 bits adds to the weights: scores of at most 64 in magnitude whose products are summed in chains of at
most 12 (error 12 * 64 * 2^-24 < 2^-14 of a weight), once in the numerator and once in the sum, and the weights' pairs (2^-16 in bf16, 2^-21 in f16): under 2^-12 of sum(weight * |value|).  Where there are many rows a weight is one
number of the type, off by up to half a step of it, which is asked for of calls of more than 16 rows and heads of a kv head.  Half a step: a type of p significant bits has numbers 2^(e + 1 - p) apart from 2^e to 2^(e + 1), so that
the nearest is off by up to 2^(e - p), which is 2^-p of a number of at least 2^e: 2^-8 in bf16, 2^-11 in f16, eps / 2 of both.  The sum that an output is divided by is of the weights as they were, so an output is off by
|sum(d_i w_i v_i)| / sum(w_i) <= eps / 2 * sum(weight * |value|), |d_i| <= eps / 2: half of that is too little.  (Nine keys whose weights are rounded once to bf16, all else in 64 bits: 1.067 times a bound with eps / 4 here, 0.733 with eps / 2.)
lse: 2^-14 + 2^-22 |lse|."""
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


class Setup:
    """A pool full of numbers that are none, shuffled tables, ragged sequences."""

    def __init__(self, pv, prefix, rows, heads=2, hd=64, pt=16, seed=0, dtype="bf16", fill=float("nan"), extra_pages=1, tail_rows=0):
        r = self.r = np.random.default_rng(seed)
        self.pv, self.prefix, self.rows, self.heads, self.hd, self.dtype = pv, list(prefix), list(rows), heads, hd, TYPES[dtype]
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.start[-1]) + tail_rows
        pages = max(1, max(-(-(p + w) // pt) for p, w in zip(prefix, rows)))
        total = pages * len(rows) + extra_pages
        self.tables = r.permutation(total)[: pages * len(rows)].reshape(len(rows), pages).astype(np.int32)
        self.pool = pv.KV16Pool(total, heads, hd, pt, dtype=self.dtype)
        self.pool.pages.fill_(fill)
        self.ref = ref.Pool(np.full((total, heads, 2, pt * hd), fill), hd, pt)

    def seqs(self, start=None, prefix=None, tables=None):
        return self.pv.KVSeqs(dev(self.start if start is None else start), dev(self.prefix if prefix is None else prefix), dev(self.tables if tables is None else tables))

    def draw(self, n, dtype=None, size=1.0):
        return torch.from_numpy(self.r.normal(size=(n, self.heads, self.hd)) * size).to(self.dtype if dtype is None else TYPES[dtype])

    def put(self, start, prefix, k, v):
        self.pool.append(self.seqs(start, prefix), k.cuda(), v.cuda())
        self.ref.append(start, prefix, self.tables, k.to(self.dtype).double().numpy(), v.to(self.dtype).double().numpy())

    def fill_prefix(self, size=0.5):
        start = np.concatenate([[0], np.cumsum(self.prefix)]).astype(np.int32)
        if start[-1]:
            self.put(start, [0] * len(self.prefix), self.draw(int(start[-1]), size=size), self.draw(int(start[-1])))

    def fill_rows(self, size=0.5):
        self.put(self.start, self.prefix, self.draw(self.n, size=size), self.draw(self.n))

    def same(self):
        got, want = self.pool.pages.double().cpu().numpy(), self.ref.pages
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


APPENDS = [([0], [1], 16), ([5], [1], 16), ([15], [1], 16), ([15], [2], 16), ([0], [16], 16), ([3], [40], 16), ([2], [2], 16), ([1], [3], 32), ([100], [77], 64), ([0, 7, 31, 16], [5, 0, 17, 1], 16),
           ([13] * 70, [1] * 70, 16), ([9, 250], [600, 33], 128), ([6] * 9, [2] * 9, 16)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("given,kept", [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("prefix,rows,pt", APPENDS)
def test_append(pv, prefix, rows, pt, given, kept, hd):
    s = Setup(pv, prefix, rows, hd=hd, pt=pt, heads=3, dtype=kept, tail_rows=2)
    s.fill_prefix()
    s.same()
    s.put(s.start, s.prefix, s.draw(s.n, given), s.draw(s.n, given))
    s.same()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("given,kept,hd,part", [("bf16", "bf16", 128, 128), ("f32", "f16", 64, 32), ("f16", "bf16", 128, 16), ("f32", "bf16", 64, 64), ("bf16", "bf16", 128, 112)])
@pytest.mark.parametrize("prefix,rows,pt,heads", [([0], [1], 16, 1), ([999], [1], 16, 8), ([5, 0, 40], [3, 0, 21], 16, 6), ([13] * 70, [1] * 70, 16, 2), ([31], [150], 32, 32)])
def test_append_rotates_keys_and_queries(pv, prefix, rows, pt, heads, given, kept, hd, part, interleaved):
    s = Setup(pv, prefix, rows, hd=hd, pt=pt, heads=2, dtype=kept, tail_rows=1)
    s.fill_prefix()
    base, amplitude = 10000.0, 1.125
    freq = [base ** (-2 * i / part) for i in range(part // 2)]
    turns = torch.tensor([f / (2 * np.pi) for f in freq], dtype=torch.float64, device="cuda")
    rot = pv.Rotary(hd, rotary_dim=part, interleaved=interleaved, turns=turns, amplitude=amplitude)
    k, v, q = s.draw(s.n, given), s.draw(s.n, given), torch.from_numpy(s.r.normal(size=(s.n, heads, hd))).to(TYPES[given])
    own = np.concatenate([np.arange(p, p + w) for p, w in zip(prefix, rows)] + [[0]])
    for positions in (None, s.r.integers(-5, 70000, s.n).astype(np.int32)):
        at = own if positions is None else positions
        into = torch.full((s.n, heads, hd), 7.0, dtype=TYPES[given], device="cuda")
        got = s.pool.append(s.seqs(), k.cuda(), v.cuda(), rotary=rot, positions=None if positions is None else dev(positions), q=q.cuda(), q_out=into)
        assert got is into and (got[-1] == 7).all()                       # the row of no sequence
        turn = lambda x: ref.turned(x.double().numpy(), at, freq, part, interleaved, amplitude)  # noqa: E731
        e = np.arange(part // 2)
        a, b = (2 * e, 2 * e + 1) if interleaved else (e, e + part // 2)

        def bound(x, want, dtype):
            size = np.zeros(want.shape)
            size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
            return torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -21 * amplitude * size + torch.finfo(dtype).tiny
        want = turn(q)
        assert (np.abs(got.double().cpu().numpy() - want) <= bound(q.double().numpy(), want, TYPES[given]))[:-1].all()
        # what was stored of the keys, then the rest of the pool as it has to be
        want = turn(k)
        off = bound(k.double().numpy(), want, s.dtype)
        now = ref.Pool(s.pool.pages.double().cpu().numpy(), hd, pt)
        stored = np.zeros(want.shape)
        for i in range(len(rows)):
            for j in range(rows[i]):
                row = s.start[i] + j
                stored[row] = now.token(s.tables[i], prefix[i] + j, 0)
                assert (np.abs(stored[row] - want[row]) <= off[row]).all()
        s.ref.append(s.start, s.prefix, s.tables, stored, v.to(s.dtype).double().numpy())
        s.same()
    # over the queries themselves, and as rotate() would have it
    mine = q.cuda()
    assert s.pool.append(s.seqs(), k.cuda(), v.cuda(), rotary=rot, q=mine, q_out=mine) is mine
    assert torch.equal(mine[:-1], rot.rotate(q.cuda(), dev(own))[:-1]) and torch.equal(mine[-1].cpu(), q[-1])


def test_every_number_of_16_bits(pv):
    """All bit patterns of both types come back as they were (NaN as some NaN), and 32-bit ones between them are rounded to nearest, ties to even."""
    for dtype in ("bf16", "f16"):
        bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[dtype]).view(512, 2, 64)
        s = Setup(pv, [0], [512], hd=64, dtype=dtype)
        s.put(s.start, [0], bits, bits.flip(0))
        s.same()
        f = bits.float()
        near = torch.where(torch.isfinite(f), f * (1 + 2.0 ** -9 * torch.randint(-3, 4, f.shape)), f)
        s.put(s.start, [0], near, -near)
        s.same()


def test_rows_in_strided_tensors_and_a_stale_tail(pv):
    s = Setup(pv, [21], [30])
    s.fill_prefix()
    fused = torch.randn(30, 6 * 64, dtype=torch.bfloat16)
    g = fused.cuda()
    view = lambda x, i: x[:, i * 128:(i + 1) * 128].view(30, 2, 64)  # noqa: E731
    s.pool.append(s.seqs(), view(g, 1), view(g, 2))
    s.ref.append(s.start, s.prefix, s.tables, view(fused, 1).double().numpy(), view(fused, 2).double().numpy())
    s.same()
    heads_first = torch.randn(2, 5, 64, dtype=torch.bfloat16)
    h = heads_first.cuda().transpose(0, 1)
    s.pool.append(s.seqs([0, 5], [24]), h, h)                            # the tokens from 29 on stay what they were
    s.ref.append([0, 5], [24], s.tables, heads_first.transpose(0, 1).double().numpy(), heads_first.transpose(0, 1).double().numpy())
    s.same()


def bad_tables(s):
    """Pages that are none, a sequence with a negative length, one whose rows run over the table's end."""
    t = s.tables.copy()
    t[0, 1], t[1, 0], t[2, -1] = -1, s.pool.n_pages, 1 << 30
    prefix = list(s.prefix)
    prefix[3] = -4
    prefix[4] = t.shape[1] * 16 - 3
    return t, prefix


@pytest.mark.parametrize("hd", [64, 128])
def test_pages_and_lengths_that_do_not_exist(pv, hd):
    s = Setup(pv, [20, 9, 30, 3, 3, 8], [17, 3, 8, 5, 9, 2], hd=hd, tail_rows=3)
    s.fill_prefix()
    t, prefix = bad_tables(s)
    k, v = s.draw(s.n), s.draw(s.n)
    seqs = s.seqs(prefix=prefix, tables=t)
    rot = pv.Rotary(hd)
    q = torch.from_numpy(s.r.normal(size=(s.n, 4, hd))).to(s.dtype)
    s.pool.append(seqs, k.cuda(), v.cuda())
    start = s.start.copy()

    def rows_of(prefix):                                                  # (the oracle takes no negative length)
        return [(i, p, start[i], start[i + 1]) for i, p in enumerate(prefix) if p >= 0]
    for i, p, a, b in rows_of(prefix):
        s.ref.append([a, b], [p], [t[i]], k.double().numpy(), v.double().numpy())
    s.same()
    turned = torch.full((s.n, 4, hd), 7.0, dtype=s.dtype, device="cuda")
    s.pool.append(seqs, k.cuda(), v.cuda(), rotary=rot, q=q.cuda(), q_out=turned)
    there = np.zeros(s.n, bool)
    for i, p, a, b in rows_of(prefix):
        there[a:b] = True
    assert (turned[torch.from_numpy(~there).cuda()] == 7).all() and (turned[torch.from_numpy(there).cuda()] != 7).any()
    s.pool.append(seqs, k.cuda(), v.cuda())
    s.same()
    for masks in (None, s.r.integers(0, 2 ** 63, (s.n, 1)).astype(np.int64)):
        out, lse = torch.full((s.n, 4, hd), 7.0, dtype=s.dtype, device="cuda"), torch.full((s.n, 4), 7.0, device="cuda")
        s.pool.attention(seqs, q.cuda(), mask=None if masks is None else dev(masks, torch.int64), out=out, lse=lse)
        assert (out[torch.from_numpy(~there).cuda()] == 7).all() and (lse[torch.from_numpy(~there).cuda()] == 7).all()
        for i, p, a, b in rows_of(prefix):
            m = None if masks is None else [int(x) for x in masks[a:b, 0].view(np.uint64)]
            check(s.ref, [0, b - a], [p], [t[i]], q[a:b], out[a:b], lse[a:b], masks=m)
    path, accepted = np.full(s.n, -1), [3, 2, 4, 3, 8, 1]
    for i in range(6):
        path[start[i]:start[i + 1]] = np.arange(start[i + 1] - start[i]) + 1
    s.pool.keep(seqs, dev(path), dev(accepted))
    for i, p, a, b in rows_of(prefix):
        s.ref.keep([0, b - a], [p], [t[i]], path[a:b], [accepted[i]])
    s.same()


@pytest.mark.parametrize("rows", [1, 9, 40])
def test_lengths_up_to_the_largest(pv, rows):
    """Rows behind a table's end are no tokens, wherever they begin; all that exist are seen.  Tables without pages: nothing is."""
    s = Setup(pv, [64 - rows], [rows], hd=128)
    s.fill_prefix()
    s.fill_rows()
    before = s.pool.pages.clone()
    q = torch.from_numpy(s.r.normal(size=(rows, 8, 128))).to(torch.bfloat16).cuda()
    masks = dev(s.r.integers(0, 2 ** 63, rows), torch.int64)
    for mask in (None, masks):
        want = s.pool.attention(s.seqs(prefix=[64]), q, mask=mask, return_lse=True)
        assert torch.isfinite(want[1]).all()
        for far in (2 ** 30, 2 ** 31 - 1 - rows, 2 ** 31 - 2, 2 ** 31 - 1):
            got = s.pool.attention(s.seqs(prefix=[far]), q, mask=mask, return_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), far
            s.pool.append(s.seqs(prefix=[far]), s.draw(rows).cuda(), s.draw(rows).cuda())
            s.pool.keep(s.seqs(prefix=[far]), torch.arange(1, rows + 1, dtype=torch.int32, device="cuda"), dev([rows]))
    none = s.seqs(tables=np.zeros((1, 0), np.int32))
    out, lse = s.pool.attention(none, q, return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    s.pool.append(none, s.draw(rows).cuda(), s.draw(rows).cuda())
    s.pool.keep(none, torch.arange(1, rows + 1, dtype=torch.int32, device="cuda"), dev([rows]))
    assert torch.equal(torch.nan_to_num(s.pool.pages), torch.nan_to_num(before))


def check(pool, start, prefix, tables, q, out, lse, scale=None, masks=None):
    many = max(b - a for a, b in zip(start, start[1:])) * q.shape[1] // pool.pages.shape[1] > 16
    scale = 1 / np.sqrt(q.shape[2]) if scale is None else scale
    want, wlse, mag = pool.attention(start, prefix, tables, q.double().cpu().numpy(), scale, masks)
    got, glse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(glse), np.isnan(wlse))     # (tokens nobody wrote may be NaN)
    none, fine, far = np.isneginf(wlse), np.isfinite(want), np.isfinite(wlse)
    assert np.isfinite(got[fine]).all() and np.array_equal(np.isneginf(glse), none) and (got[none] == 0).all()
    bound = torch.finfo(out.dtype).eps / 2 * np.abs(want) + (2.0 ** -12 + many * torch.finfo(out.dtype).eps / 2) * mag + torch.finfo(out.dtype).tiny
    worst = (np.abs(got - want) / bound)[fine].max() if fine.any() else 0
    assert worst <= 1, worst
    assert (np.abs(glse[far] - wlse[far]) <= 2.0 ** -14 + 2.0 ** -22 * np.abs(wlse[far])).all()


# prefix, rows, kv heads, query heads, page
ATTEND = [([0], [1], 1, 1, 16), ([1], [1], 2, 8, 16), ([15], [1], 2, 2, 16), ([31], [1], 1, 4, 16), ([63], [1], 1, 4, 16), ([64], [2], 2, 8, 16), ([255], [3], 1, 8, 16), ([300], [8], 2, 8, 64),
          ([700], [1], 1, 5, 16), ([1100], [4], 2, 4, 16), ([0], [17], 2, 8, 16), ([0], [130], 1, 4, 16), ([77], [65], 2, 6, 32), ([513], [33], 1, 16, 16),
          ([0, 40, 0, 511, 1000], [3, 0, 1, 9, 1], 2, 8, 16), ([5] * 70, [1] * 70, 1, 2, 16), ([200, 0, 31], [1, 100, 40], 2, 8, 16), ([3000], [2], 1, 4, 16), ([90], [5], 1, 70, 16)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("prefix,rows,kvh,heads,pt", ATTEND)
def test_attention(pv, prefix, rows, kvh, heads, pt, dtype, hd):
    s = Setup(pv, prefix, rows, heads=kvh, hd=hd, pt=pt, dtype=dtype, tail_rows=1)
    s.fill_prefix()
    s.fill_rows()
    q = torch.from_numpy(s.r.normal(size=(s.n, heads, hd))).to(TYPES[dtype])
    out, lse = torch.full((s.n, heads, hd), 7.0, dtype=q.dtype, device="cuda"), torch.full((s.n, heads), 7.0, device="cuda")
    s.pool.attention(s.seqs(), q.cuda(), out=out, lse=lse)
    assert (out[-1] == 7).all() and (lse[-1] == 7).all()
    check(s.ref, s.start, s.prefix, s.tables, q[:-1], out[:-1], lse[:-1])


def random_masks(s, words, r):
    m = r.integers(0, 2 ** 63, (s.n, words)).astype(np.int64)
    m[0], m[-1], m[s.n // 2] = 0, -1, 1
    whole = [sum(int(w) << (64 * i) for i, w in enumerate(row.view(np.uint64))) for row in m]
    return m, whole


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("f16", 128), ("bf16", 128)])
@pytest.mark.parametrize("prefix,rows,words", [([100], [48], 1), ([0], [7], 1), ([300, 0, 17], [64, 5, 20], 1), ([50], [70], 1), ([0], [65], 2), ([50], [70], 2), ([1000], [150], 3), ([31, 0, 64], [129, 128, 3], 3),
                                               ([20], [200], 2), ([5], [9], 4), ([2000], [300], 5)])
def test_attention_with_masks(pv, prefix, rows, words, dtype, hd):
    """Rows that see nothing of the block, rows that see nothing at all, slots that the mask has no bit for, words behind the rows."""
    s = Setup(pv, prefix, rows, heads=2, hd=hd, dtype=dtype)
    s.fill_prefix()
    s.fill_rows()
    m, whole = random_masks(s, words, s.r)
    q = torch.from_numpy(s.r.normal(size=(s.n, 8, hd))).to(TYPES[dtype])
    out, lse = s.pool.attention(s.seqs(), q.cuda(), mask=dev(m[:, 0] if words == 1 else m, torch.int64), return_lse=True)
    check(s.ref, s.start, s.prefix, s.tables, q, out, lse, masks=whole)


def test_a_mask_of_a_chain_is_no_mask(pv):
    for rows in (5, 90):
        s = Setup(pv, [77], [rows], heads=2, hd=128)
        s.fill_prefix()
        s.fill_rows()
        q = torch.from_numpy(s.r.normal(size=(rows, 8, 128))).to(torch.bfloat16).cuda()
        m = np.array([[((1 << (i + 1)) - 1) >> (64 * w) & (2 ** 64 - 1) for w in range(2)] for i in range(rows)], dtype=np.uint64).view(np.int64)
        a, b = s.pool.attention(s.seqs(), q, return_lse=True), s.pool.attention(s.seqs(), q, mask=dev(m, torch.int64), return_lse=True)
        assert (a[0].float() - b[0].float()).abs().max() <= 2.0 ** -7 * a[0].float().abs().max() and (a[1] - b[1]).abs().max() <= 2.0 ** -14


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales(pv, dtype):
    """Scores far apart, equal ones, none (a scale of 0), and a negative scale."""
    for rows in (2, 70):
        s = Setup(pv, [400], [rows], heads=1, hd=64, dtype=dtype)
        k, v = torch.randn(400 + rows, 1, 64) * 0.1, torch.randn(400 + rows, 1, 64)
        k[0], v[0] = 1.0, 1e-3
        start = [0, 400 + rows]
        s.put(start, [0], k.to(s.dtype), v.to(s.dtype))
        for scale in (0.0, 0.02, 0.9, -0.02, -0.9):
            q = (torch.ones(rows, 2, 64) * torch.tensor([1.0, 0.5]).view(1, 2, 1)).to(s.dtype)
            out, lse = s.pool.attention(s.seqs(), q.cuda(), scale=scale, return_lse=True)
            check(s.ref, s.start, s.prefix, s.tables, q, out, lse, scale=scale)


def test_many_small_weights_beside_a_large_one(pv):
    """20000 keys of 2^-17 of the first one's weight each: more than an f16 weight of 1 can hold beside it."""
    for dtype in ("bf16", "f16"):
        s = Setup(pv, [20000], [1], heads=1, hd=64, dtype=dtype)
        k, v = torch.zeros(20001, 1, 64), torch.ones(20001, 1, 64)
        k[0, 0, 0], v[0] = 17 * np.log(2), 0.0
        s.put([0, 20001], [0], k.to(s.dtype), v.to(s.dtype))
        q = torch.zeros(1, 1, 64)
        q[0, 0, 0] = 1
        out, lse = s.pool.attention(s.seqs(), q.to(s.dtype).cuda(), scale=1.0, return_lse=True)
        check(s.ref, s.start, s.prefix, s.tables, q, out, lse, scale=1.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows,prefix", [(8, 90), (70, 90), (70, 64), (40, 0), (33, 31)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_a_row_does_not_see_has_no_influence(pv, bad, rows, prefix, dtype):
    """Not finite keys and values in the block: rows that see them are not finite (of a value: in its feature), the others what they are without them."""
    s = Setup(pv, [prefix], [rows], heads=1, hd=64, dtype=dtype)
    s.fill_prefix()
    k, v = s.draw(rows, size=0.5), s.draw(rows)
    q = torch.from_numpy(s.r.normal(size=(rows, 4, 64))).to(s.dtype)
    masks = [((1 << rows) - 1) & ~(1 << 5) if i % 3 else (1 << rows) - 1 for i in range(rows)]
    words = -(-rows // 64)
    m = np.array([[x >> (64 * w) & (2 ** 64 - 1) for w in range(words)] for x in masks], dtype=np.uint64).view(np.int64)
    for mask, sees in ((None, torch.arange(rows) >= 5), (dev(m, torch.int64), torch.arange(rows) % 3 == 0)):
        s.pool.append(s.seqs(), k.cuda(), v.cuda())
        clean = s.pool.attention(s.seqs(), q.cuda(), mask=mask).cpu()
        for which in ("k", "v"):
            kk, vv = k.clone(), v.clone()
            (kk if which == "k" else vv)[5, 0, 9] = bad
            s.pool.append(s.seqs(), kk.cuda(), vv.cuda())
            out = s.pool.attention(s.seqs(), q.cuda(), mask=mask).cpu()
            assert torch.equal(out[~sees], clean[~sees])
            if which == "v":
                f = torch.arange(64) == 9
                assert torch.equal(out[..., ~f], clean[..., ~f])
                # (a weight is a pair of numbers, the second of either sign or 0: infinity times the pair is infinity, or infinity less infinity, or infinity times 0, NaN)
                there = out[sees][..., 9]
                assert there.isnan().all() if bad != bad else (there.isnan() | (there == bad)).all()
            elif bad != bad:
                assert out[sees].isnan().all()


def test_both_infinities_make_nan_and_tokens_behind_the_end_do_not_matter(pv):
    s = Setup(pv, [40], [20], heads=1, hd=64)                             # (the pool is full of NaN behind the rows)
    s.fill_prefix()
    k, v = s.draw(20), s.draw(20)
    v[3, 0, 7], v[9, 0, 7], v[9, 0, 8] = float("inf"), -float("inf"), float("inf")
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    q = torch.randn(20, 2, 64, dtype=torch.bfloat16)
    out = s.pool.attention(s.seqs(), q.cuda()).cpu()
    assert torch.isfinite(out[:3]).all() and torch.isfinite(out[..., :7]).all() and torch.isfinite(out[..., 9:]).all() and torch.isfinite(out[:9, :, 8]).all()
    assert not torch.isfinite(out[3:, :, 7]).any() and out[9:, :, 7].isnan().all() and not torch.isfinite(out[9:, :, 8]).any()


def test_strides_in_place_and_graphs(pv):
    """q as a slice of a fused projection, the result over it; one graph replayed after lengths, tables and data have changed; beside it another graph of the same shapes."""
    s = Setup(pv, [1500, 700], [3, 2], heads=2, hd=64)
    s.fill_prefix()
    s.fill_rows()
    fused = torch.randn(5, 12 * 64, dtype=torch.bfloat16, device="cuda")
    q = fused[:, :512].view(5, 8, 64)
    seqs = s.seqs()
    want = s.pool.attention(seqs, q.contiguous())
    rest = fused[:, 512:].clone()
    graphs, outs = [], []
    for i in range(2):
        outs.append(torch.empty(5, 8, 64, dtype=torch.bfloat16, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.pool.attention(seqs, q, out=outs[-1])
    for i in range(3):
        seqs.prefix_len.copy_(dev([1500 - 100 * i, 3 + i]))
        for g in graphs:
            g.replay()
        fresh = s.pool.attention(seqs, q.contiguous())
        assert torch.equal(outs[0], fresh) and torch.equal(outs[1], fresh)
    seqs.prefix_len.copy_(dev([1500, 700]))
    assert s.pool.attention(seqs, q, out=q).data_ptr() == q.data_ptr()
    assert torch.equal(q, want) and torch.equal(fused[:, 512:], rest)


def test_another_stream(pv):
    s = Setup(pv, [3000], [4], heads=2, hd=128)
    s.fill_prefix()
    s.fill_rows()
    q = torch.randn(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    want = s.pool.attention(s.seqs(), q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [s.pool.attention(s.seqs(), q, stream=side) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(g, want) for g in got)


def test_places_past_4_gib(pv):
    """Pages whose bytes lie beyond 2^32 (filled to the end: what nobody wrote differs between two pools)."""
    n = 70000
    pool = pv.KV16Pool(n, 8, 128)                                         # 4.6 GB
    far = torch.tensor([[n - 1, 3, n - 2]], dtype=torch.int32, device="cuda")
    seqs, small = pv.KVSeqs(dev([0, 48]), dev([0]), far), pv.KV16Pool(4, 8, 128)
    near = pv.KVSeqs(dev([0, 48]), dev([0]), dev([[0, 1, 2]]))
    k, v, q = (torch.randn(48, h, 128, dtype=torch.bfloat16, device="cuda") for h in (8, 8, 32))
    for p, x in ((pool, seqs), (small, near)):
        p.append(x, k, v)
    assert torch.equal(pool.attention(seqs, q), small.attention(near, q))
    path, one = torch.arange(10, 58, dtype=torch.int32, device="cuda"), dev([20])
    pool.keep(seqs, path, one); small.keep(near, path, one)
    assert torch.equal(pool.pages[[n - 1, 3, n - 2]], small.pages[:3])


KEEPS = [([0], [1], [0], 16), ([5], [2], [1], 16), ([14], [9], [4], 16), ([100], [48], [6], 64), ([3, 0, 61, 16], [17, 0, 24, 1], [9, 3, 23, 0], 16), ([250], [300], [140], 32), ([7] * 20, [12] * 20, [3] * 20, 16)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("prefix,rows,accepted,pt", KEEPS)
def test_keep(pv, prefix, rows, accepted, pt, hd):
    """Paths that begin with the tree's first rows, that skip some, that reach the last; what follows is left as it was."""
    for seed in range(4):
        s = Setup(pv, prefix, rows, heads=3, hd=hd, pt=pt, seed=seed, tail_rows=1)
        s.fill_prefix()
        s.fill_rows()
        path = np.full(s.n, -1)
        for i, (r, a) in enumerate(zip(rows, accepted)):
            if r:
                a = min(a, r - 1)
                path[s.start[i]:s.start[i] + a + 1] = [0] + sorted(s.r.choice(np.arange(1, r), a, replace=False).tolist()) if r > 1 else [0]
        s.pool.keep(s.seqs(), dev(path), dev(accepted))
        s.ref.keep(s.start, s.prefix, s.tables, path, accepted)
        s.same()


def test_keep_of_numbers_that_are_no_rows(pv):
    s = Setup(pv, [9], [20], heads=2, hd=64)
    s.fill_prefix()
    s.fill_rows()
    path = np.arange(20) - 1                                              # less than their places
    path[3], path[6], path[8], path[9] = 20, 2 ** 31 - 1, -2 ** 31, 15
    for accepted in (-1, -2 ** 31, 0, 2 ** 31 - 1):
        s.pool.keep(s.seqs(), dev(path), dev([accepted]))
        s.ref.keep(s.start, s.prefix, s.tables, path, [accepted])
        s.same()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_steps_of_a_tree(pv, dtype):
    """As a program uses them together: drafts of a tree appended with their rotary positions, attended to, verified, the path kept, three steps in a row; in the end the cache holds what a chain of the accepted tokens
    appended at once leaves, and attention over it is the oracle's."""
    r = np.random.default_rng(11)
    hd, kvh, heads, vocab, n_seq, steps = 64, 2, 8, 97, 3, 3
    embed = torch.from_numpy(r.normal(size=(vocab, kvh + kvh + heads, hd)) * 0.5).to(TYPES[dtype]).cuda()
    unembed = torch.from_numpy(r.normal(size=(heads * hd, vocab)) * 0.3).float().cuda()
    pages = 8
    table = torch.from_numpy(r.permutation(pages * n_seq).reshape(n_seq, pages).astype(np.int32)).cuda()
    pool, chain = (pv.KV16Pool(pages * n_seq, kvh, hd, dtype=TYPES[dtype]) for _ in range(2))
    rot = pv.Rotary(hd, base=500.0)
    prefix = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    history = [[int(r.integers(vocab))] for _ in range(n_seq)]            # the last token of each is not in the cache yet
    for step in range(steps):
        sizes = [int(r.integers(3, 30)) for _ in range(n_seq)]
        start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        tokens, parent, depth, masks = [], [], [], []
        for i, m in enumerate(sizes):
            mine = [0]
            for j in range(m):
                up = -1 if j == 0 else int(r.integers(0, j))
                parent.append(up)
                depth.append(0 if j == 0 else depth[start[i] + up] + 1)
                masks.append((1 << j) | (masks[start[i] + up] if j else 0))
                tokens.append(history[i][-1] if j == 0 else int(r.integers(vocab)))
        tokens_d, parent_d = dev(tokens), dev(parent)
        seqs = pv.KVSeqs(dev(start), prefix, table)
        positions = (prefix.repeat_interleave(dev(sizes).long()) + dev(depth)).to(torch.int32)
        x = embed[tokens_d.long()]
        q = pool.append(seqs, x[:, :kvh], x[:, kvh:2 * kvh], rotary=rot, positions=positions, q=x[:, 2 * kvh:])
        out = pool.attention(seqs, q, mask=dev(np.array(masks, dtype=np.int64), torch.int64))
        logits = out.float().reshape(len(tokens), -1) @ unembed
        u = torch.from_numpy(r.random((len(tokens), 2))).cuda()
        got = pv.verify_drafts(dev(start), logits, tokens_d, u, parent=parent_d, temperature=1.0)
        a, f, path, _ = ref.verify(start, logits.double().cpu().numpy(), np.array(tokens), u.cpu().numpy(), [1.0] * n_seq, None, np.array(parent))
        assert got.accepted.tolist() == a.tolist() and got.next_token.tolist() == f.tolist() and got.path.tolist() == path.tolist()
        pool.keep(seqs, got.path, got.accepted)
        prefix = prefix + got.accepted + 1
        for i in range(n_seq):
            for d in range(1, int(a[i]) + 1):
                history[i].append(tokens[start[i] + path[start[i] + d]])
            history[i].append(int(f[i]))
    assert [len(h) - 1 for h in history] == prefix.tolist()
    sizes = prefix.tolist()
    start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    x = embed[dev(sum([h[:-1] for h in history], [])).long()]
    seqs = pv.KVSeqs(dev(start), dev([0] * n_seq), table)
    q = chain.append(seqs, x[:, :kvh], x[:, kvh:2 * kvh], rotary=rot, q=x[:, 2 * kvh:])
    a, b = ref.Pool(pool.pages.double().cpu().numpy(), hd, 16), ref.Pool(chain.pages.double().cpu().numpy(), hd, 16)
    for i in range(n_seq):
        for t in range(sizes[i]):
            for which in (0, 1):
                assert np.array_equal(a.token(table[i].tolist(), t, which), b.token(table[i].tolist(), t, which))
    out, lse = pool.attention(seqs, q, return_lse=True)
    check(a, start, [0] * n_seq, table.tolist(), q, out, lse)
