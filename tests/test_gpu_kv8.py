"""The operators of the 8-bit key/value cache against the 64-bit oracle (tests/kv8_ref.py).

Codes and scales have to be equal, byte for byte, in the whole pool.  Attention: a bf16 (f16) output is off by half a step, eps / 2 of its value, plus what the
arithmetic in 32 bits adds to the weights: scores of at most 64 in magnitude whose products are summed in chains of at most 12 (error 12 * 64 * 2^-24 < 2^-14 of a weight), once in
the numerator and once in the sum: under 2^-12 of sum(weight * |value|).  For f16 outputs the weights are a pair of f16 (2^-22, in that); for bf16 outputs they are one f16, each off by up to
half a step of it, 2^-11, in the numerator: 2^-11 of sum(weight * |value|) more.  lse: 2^-14 + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

import kv8_ref as ref

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
    """A pool full of bytes that mean nothing, shuffled tables, ragged sequences."""
    room = 0                                                              # pages that no sequence has, behind those of its table

    def __init__(self, pv, prefix, rows, heads=2, hd=64, pt=16, seed=0, fill=0xFF, extra_pages=1, tail_rows=0):
        r = self.r = np.random.default_rng(seed)
        self.prefix, self.rows, self.heads, self.hd = list(prefix), list(rows), heads, hd
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.start[-1]) + tail_rows
        pages = max(1, max(-(-(p + w) // pt) for p, w in zip(prefix, rows)))
        total = pages * len(rows) + extra_pages
        self.tables = r.permutation(total)[: pages * len(rows)].reshape(len(rows), pages).astype(np.int32)
        self.pool = pv.KV8Pool(total, heads, hd, pt)
        self.pool.codes.fill_(fill)
        self.pool.scales.fill_(fill)
        self.ref = ref.Pool(np.full((total, heads, 2, pt * hd), fill, np.uint8), np.full((total, heads, pt // 16, 2), fill, np.uint8), hd, pt)
        self.pv = pv

    def seqs(self, start=None, prefix=None, tables=None):
        tables = np.asarray(self.tables if tables is None else tables)
        tables = np.concatenate([tables, np.full((tables.shape[0], self.room), -1, tables.dtype)], axis=1)
        return self.pv.KV8Seqs(dev(self.start if start is None else start), dev(self.prefix if prefix is None else prefix), dev(tables))

    def draw(self, n, dtype, spread=2.0):
        x = torch.from_numpy(self.r.normal(size=(n, self.heads, self.hd)) * 2.0 ** self.r.uniform(-spread, spread, size=(n, self.heads, 1))).to(TYPES[dtype])
        return x

    def fill_prefix(self, dtype="bf16"):
        """The tokens before the rows: written through the library, and by the oracle."""
        start = np.concatenate([[0], np.cumsum(self.prefix)]).astype(np.int32)
        n = int(start[-1])
        if n:
            k, v = self.draw(n, dtype), self.draw(n, dtype)
            zero = [0] * len(self.prefix)
            self.pool.append(self.seqs(start, zero), k.cuda(), v.cuda())
            self.ref.append(start, zero, self.tables, k.double().numpy(), v.double().numpy())

    def same(self):
        assert np.array_equal(self.pool.scales.cpu().numpy(), self.ref.scales)
        assert np.array_equal(self.pool.codes.cpu().numpy(), self.ref.codes)


APPENDS = [([0], [1], 16), ([5], [1], 16), ([15], [1], 16), ([15], [2], 16), ([0], [16], 16), ([3], [40], 16), ([100], [77], 64), ([0, 7, 31, 16], [5, 0, 17, 1], 16),
           ([13] * 70, [1] * 70, 16), ([9, 250], [600, 33], 128)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("prefix,rows,pt", APPENDS)
def test_append_and_read(pv, prefix, rows, pt, dtype, hd):
    s = Setup(pv, prefix, rows, hd=hd, pt=pt, heads=3, tail_rows=2)
    s.fill_prefix(dtype)
    s.same()
    k, v = s.draw(s.n, dtype), s.draw(s.n, dtype)
    seqs = s.seqs()
    s.pool.append(seqs, k.cuda(), v.cuda())
    s.ref.append(s.start, s.prefix, s.tables, k.double().numpy(), v.double().numpy())
    s.same()
    for out in (torch.float32, torch.bfloat16, torch.float16):
        gk, gv = (torch.full((s.n, 3, hd), 7.0, dtype=out, device="cuda") for _ in range(2))
        s.pool.read(seqs, s.n, out=(gk, gv))
        want = [np.concatenate([s.ref.tokens(t, p, n)[w] for t, p, n in zip(s.tables, s.prefix, s.rows)]) for w in (0, 1)]
        for got, w in zip((gk, gv), want):
            assert np.array_equal(got[: s.start[-1]].double().cpu().numpy(), torch.from_numpy(w).to(out).double().numpy())
            assert (got[s.start[-1]:] == 7).all()                        # rows of no sequence


@pytest.mark.parametrize("many", [False, True])
def test_a_prompt_at_once_is_the_same_for_both_walks(pv, many):
    """Few rows: a wave each; many: a wave for 16 of them, whatever blocks they lie in."""
    rows = [700, 1, 650] if many else [70, 1, 65]
    s = Setup(pv, [3, 0, 21], rows, heads=2, hd=64)
    s.fill_prefix()
    k, v = s.draw(s.n, "bf16"), s.draw(s.n, "bf16")
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    s.ref.append(s.start, s.prefix, s.tables, k.double().numpy(), v.double().numpy())
    s.same()


def test_every_bf16_number(pv):
    """All finite bf16 bit patterns, 64 to a token of its own scale block, and under the scale of one large token."""
    bits = np.arange(65536, dtype=np.uint32)
    x = (bits << 16).view(np.float32)
    x = x[np.isfinite(x)].reshape(-1, 64)
    for prefix in (0, 1):
        n = x.shape[0]
        s = Setup(pv, [prefix] * n, [1] * n, heads=1, hd=64)
        if prefix:
            big = torch.full((n, 1, 64), 100.0, dtype=torch.float32)
            s.pool.append(s.seqs(np.arange(n + 1), [0] * n), big.cuda(), big.cuda())
            s.ref.append(np.arange(n + 1), [0] * n, s.tables, big.numpy(), big.numpy())
        k = torch.from_numpy(x.reshape(n, 1, 64).copy()).to(torch.bfloat16)
        s.pool.append(s.seqs(), k.cuda(), (-k).cuda())
        s.ref.append(s.start, s.prefix, s.tables, k.double().numpy(), (-k).double().numpy())
        s.same()


def test_not_finite_zero_and_extreme_numbers(pv):
    rows = [6, 3, 20, 4]
    s = Setup(pv, [0, 5, 11, 14], rows, heads=2, hd=128)
    s.fill_prefix("f32")
    k, v = s.draw(s.n, "f32").float(), s.draw(s.n, "f32").float()
    k[0], v[1] = 0.0, 0.0
    k[6], v[7] = 0.0, -0.0
    k[2, 0, 3], k[2, 1, 5], v[3, 0, 7], v[4, 1] = float("inf"), float("nan"), float("-inf"), float("nan")
    k[10, 0], v[11, 1, 9] = 3.0e38, -3.3e38
    k[12, 1, :64], v[13, 0] = 1e-40, 1e-38
    k[14, 0, 1], v[20] = 1e9, 1e-30
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    s.ref.append(s.start, s.prefix, s.tables, k.numpy(), v.numpy())
    assert np.array_equal(s.pool.scales.cpu().numpy(), s.ref.scales)
    got, want = ref.VALUES[s.pool.codes.cpu().numpy()], ref.VALUES[s.ref.codes]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_a_block_filled_token_by_token(pv):
    """Tokens that grow and shrink, one call each: scales are raised and never lowered, and the values are those of one call but for the smallest."""
    s, t = (Setup(pv, [0], [16], heads=2, hd=64, seed=4) for _ in range(2))
    k, v = s.draw(16, "bf16", spread=6), s.draw(16, "bf16", spread=6)
    for i in range(16):
        one = s.seqs([0, 1], [i])
        s.pool.append(one, k[i:i + 1].cuda(), v[i:i + 1].cuda())
        s.ref.append([0, 1], [i], s.tables, k[i:i + 1].double().numpy(), v[i:i + 1].double().numpy())
        s.same()
    t.ref.append(t.start, [0], t.tables, k.double().numpy(), v.double().numpy())
    a, b = s.ref.tokens(s.tables[0], 0, 16), t.ref.tokens(t.tables[0], 0, 16)
    for x, y in zip(a[:2], b[:2]):
        assert np.abs(x - y).max() <= 2.0 ** -9 * np.abs(y).max() / 224 and np.array_equal(x[np.abs(y) > np.abs(y).max() / 2 ** 12], y[np.abs(y) > np.abs(y).max() / 2 ** 12])


def test_rows_in_strided_tensors_and_a_stale_tail(pv):
    """Keys and values as slices of one fused projection; heads before rows; tokens of an earlier, longer sequence behind the rows."""
    s = Setup(pv, [21], [30], heads=2, hd=64)
    s.fill_prefix()
    fused = torch.randn(30, 2 * 64 * 3, dtype=torch.bfloat16)
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
    k, v = (torch.zeros(2, 30, 64, dtype=torch.float16, device="cuda").transpose(0, 1) for _ in range(2))
    s.pool.read(s.seqs(), 30, out=(k, v))
    want = s.ref.tokens(s.tables[0], 21, 30)
    assert np.array_equal(k.double().cpu().numpy(), want[0]) and np.array_equal(v.double().cpu().numpy(), want[1])


def bad_tables(s):
    """Pages that are none, a table that ends early, a sequence with a negative length, rows of no sequence."""
    t = s.tables.copy()
    t[0, 1], t[1, 0], t[2, -1] = -1, s.pool.n_pages, 1 << 30
    prefix = list(s.prefix)
    prefix[3] = -4
    prefix[4] = t.shape[1] * 16 - 3                                       # its rows run over the table's end
    return t, prefix


def test_pages_and_lengths_that_do_not_exist(pv):
    s = Setup(pv, [20, 9, 30, 3, 3, 8], [17, 3, 8, 5, 9, 2], heads=2, hd=64, tail_rows=3)
    s.fill_prefix()
    t, prefix = bad_tables(s)
    k, v = s.draw(s.n, "bf16"), s.draw(s.n, "bf16")
    seqs = s.seqs(prefix=prefix, tables=t)
    s.pool.append(seqs, k.cuda(), v.cuda())
    s.ref.append(s.start, prefix, t, k.double().numpy(), v.double().numpy())
    s.same()
    gk, gv = (torch.full((s.n, 2, 64), 7.0, device="cuda") for _ in range(2))
    s.pool.read(seqs, s.n, out=(gk, gv))
    for i, (p, r) in enumerate(zip(prefix, s.rows)):
        part = slice(s.start[i], s.start[i] + r)
        if p < 0:
            assert (gk[part] == 7).all()
            continue
        wk, wv, _ = s.ref.tokens(t[i], p, r)
        assert np.array_equal(gk[part].double().cpu().numpy(), wk) and np.array_equal(gv[part].double().cpu().numpy(), wv)
    assert (gk[s.start[-1]:] == 7).all()
    q = torch.randn(s.n, 4, 64, dtype=torch.bfloat16)
    out = torch.full((s.n, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((s.n, 4), 7.0, device="cuda")
    s.pool.attention(seqs, q.cuda(), out=out, lse=lse)
    check_attention(s, q, out, lse, prefix=prefix, tables=t, untouched=7.0)


@pytest.mark.parametrize("rows", [1, 9, 40])
def test_lengths_up_to_the_largest(pv, rows):
    """Rows behind a table's end are no tokens, wherever they begin; all that exist are seen.  Tables without pages: nothing is."""
    s = Setup(pv, [64 - rows], [rows], heads=2, hd=128)
    s.fill_prefix()
    s.pool.append(s.seqs(), s.draw(s.n, "bf16").cuda(), s.draw(s.n, "bf16").cuda())
    before = s.pool.codes.clone()
    q = torch.from_numpy(s.r.normal(size=(rows, 8, 128))).to(torch.bfloat16).cuda()
    masks = dev(s.r.integers(0, 2 ** 63, rows), torch.int64)
    for mask in (None, masks):
        want = s.pool.attention(s.seqs(prefix=[64]), q, mask=mask, return_lse=True)
        assert torch.isfinite(want[1]).all()
        for far in (2 ** 30, 2 ** 31 - 1 - rows, 2 ** 31 - 2, 2 ** 31 - 1):
            got = s.pool.attention(s.seqs(prefix=[far]), q, mask=mask, return_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), far
            s.pool.append(s.seqs(prefix=[far]), s.draw(rows, "bf16").cuda(), s.draw(rows, "bf16").cuda())
            k, v = s.pool.read(s.seqs(prefix=[far]), rows)
            assert not k.any() and not v.any()
    assert torch.equal(s.pool.codes, before)
    none = s.seqs(tables=np.zeros((1, 0), np.int32))
    out, lse = s.pool.attention(none, q, return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    s.pool.append(none, s.draw(rows, "bf16").cuda(), s.draw(rows, "bf16").cuda())
    assert not s.pool.read(none, rows)[0].any() and torch.equal(s.pool.codes, before)


def check_attention(s, q, out, lse, scale=None, masks=None, prefix=None, tables=None, untouched=None):
    scale = 1 / np.sqrt(s.hd) if scale is None else scale
    want, wlse, mag, mine = ref.attention(s.ref, s.start, s.prefix if prefix is None else prefix, s.tables if tables is None else tables, q.double().numpy(), scale, masks)
    got, glse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    if untouched is not None:
        assert (got[~mine] == untouched).all() and (glse[~mine] == untouched).all()
    got, glse, want, wlse, mag = got[mine], glse[mine], want[mine], wlse[mine], mag[mine]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(glse), np.isnan(wlse))     # (tokens nobody wrote may be NaN)
    none, fine, far = np.isneginf(wlse), np.isfinite(want), np.isfinite(wlse)
    assert np.isfinite(got[fine]).all() and np.array_equal(np.isneginf(glse), none) and (got[none] == 0).all()
    bound = torch.finfo(q.dtype).eps / 2 * np.abs(want) + (2.0 ** -12 + (2.0 ** -11 if q.dtype == torch.bfloat16 else 0.0)) * mag + torch.finfo(q.dtype).tiny
    worst = (np.abs(got - want) / bound)[fine].max()
    assert worst <= 1, worst
    assert (np.abs(glse[far] - wlse[far]) <= 2.0 ** -14 + 2.0 ** -22 * np.abs(wlse[far])).all()


# prefix, rows, kv heads, query heads, page
ATTEND = [([0], [1], 1, 1, 16), ([1], [1], 2, 8, 16), ([15], [1], 2, 2, 16), ([63], [1], 1, 4, 16), ([64], [2], 2, 8, 16), ([255], [3], 1, 8, 16), ([300], [8], 2, 8, 64),
          ([700], [1], 1, 5, 16), ([1100], [4], 2, 4, 16), ([0], [17], 2, 8, 16), ([0], [130], 1, 4, 16), ([77], [65], 2, 6, 32), ([513], [33], 1, 16, 16),
          ([0, 40, 0, 511, 1000], [3, 0, 1, 9, 1], 2, 8, 16), ([5] * 70, [1] * 70, 1, 2, 16), ([200, 0, 31], [1, 100, 40], 2, 8, 16), ([3000], [2], 1, 4, 16), ([90], [5], 1, 70, 16)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("prefix,rows,kvh,heads,pt", ATTEND)
def test_attention(pv, prefix, rows, kvh, heads, pt, dtype, hd):
    s = Setup(pv, prefix, rows, heads=kvh, hd=hd, pt=pt, tail_rows=1)
    s.fill_prefix()
    k, v = s.draw(s.n, "bf16", 0.5), s.draw(s.n, "bf16")
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    s.ref.append(s.start, s.prefix, s.tables, k.double().numpy(), v.double().numpy())
    q = torch.from_numpy(s.r.normal(size=(s.n, heads, hd))).to(TYPES[dtype])
    out, lse = torch.full((s.n, heads, hd), 7.0, dtype=q.dtype, device="cuda"), torch.full((s.n, heads), 7.0, device="cuda")
    s.pool.attention(s.seqs(), q.cuda(), out=out, lse=lse)
    check_attention(s, q, out, lse, untouched=7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("prefix,rows", [([100], [48]), ([0], [7]), ([300, 0, 17], [64, 5, 20]), ([50], [70])])
def test_attention_with_masks(pv, prefix, rows, dtype):
    """Trees, rows that see nothing of the block, rows that see nothing at all, slots from 64 on."""
    s = Setup(pv, prefix, rows, heads=2, hd=64)
    s.fill_prefix()
    k, v = s.draw(s.n, "bf16", 0.5), s.draw(s.n, "bf16")
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    s.ref.append(s.start, s.prefix, s.tables, k.double().numpy(), v.double().numpy())
    masks = s.r.integers(0, 2 ** 63, s.n).astype(np.int64)
    masks[0], masks[-1], masks[s.n // 2] = 0, -1, 1
    q = torch.from_numpy(s.r.normal(size=(s.n, 8, 64))).to(TYPES[dtype])
    out, lse = s.pool.attention(s.seqs(), q.cuda(), mask=dev(masks, torch.int64), return_lse=True)
    check_attention(s, q, out, lse, masks=masks.view(np.uint64))


def test_scales_far_apart_and_a_weight_that_takes_nearly_all(pv):
    """Values whose scales differ by 2^40; a first token that takes all but 1e-6 of the weight, with values of nearly nothing."""
    s = Setup(pv, [400], [2], heads=1, hd=64)
    k, v = torch.randn(402, 1, 64) * 0.1, torch.randn(402, 1, 64)
    v[:200] *= 2.0 ** -20
    v[200:216] *= 2.0 ** 20
    k[200:216] = -k[0] * 100                                              # the huge values' keys: no weight to speak of
    k[0], v[0] = 3.0, 1e-12
    start = [0, 402]
    s.pool.append(s.seqs(start, [0]), k.cuda(), v.cuda())
    s.ref.append(start, [0], s.tables, k.double().numpy(), v.double().numpy())
    for scale in (0.02, 0.07, -0.02):
        q = (torch.ones(2, 2, 64) * torch.tensor([1.0, 0.5]).view(1, 2, 1)).to(torch.bfloat16)
        out, lse = s.pool.attention(s.seqs(), q.cuda(), scale=scale, return_lse=True)
        check_attention(s, q, out, lse, scale=scale)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [8, 70])
def test_what_a_row_does_not_see_has_no_influence(pv, bad, rows):
    """Not finite keys and values in the block: rows that see them are NaN, the others what they are without them."""
    s = Setup(pv, [90], [rows], heads=1, hd=64)
    s.fill_prefix()
    k, v = s.draw(rows, "bf16", 0.5), s.draw(rows, "bf16")
    q = torch.from_numpy(s.r.normal(size=(rows, 4, 64))).to(torch.bfloat16)
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    clean = s.pool.attention(s.seqs(), q.cuda())
    for which in ("k", "v"):
        kk, vv = k.clone(), v.clone()
        (kk if which == "k" else vv)[5, 0, 9] = bad
        s.pool.append(s.seqs(), kk.cuda(), vv.cuda())
        out = s.pool.attention(s.seqs(), q.cuda())
        assert torch.equal(out[:5], clean[:5])
        if which == "k":
            assert out[5:].isnan().all()
        else:
            assert out[5:, :, 9].isnan().all() and torch.equal(out[5:, :, :9], clean[5:, :, :9]) and torch.equal(out[5:, :, 10:], clean[5:, :, 10:])
        masks = torch.full((rows,), 0b11011111, dtype=torch.int64, device="cuda")
        masked = s.pool.attention(s.seqs(), q.cuda(), mask=masks)
        s.pool.append(s.seqs(), k.cuda(), v.cuda())
        assert torch.equal(masked, s.pool.attention(s.seqs(), q.cuda(), mask=masks))


def test_in_place_and_strided_queries(pv):
    s = Setup(pv, [600, 30], [3, 20], heads=2, hd=64)
    s.fill_prefix()
    k, v = s.draw(s.n, "bf16", 0.5), s.draw(s.n, "bf16")
    s.pool.append(s.seqs(), k.cuda(), v.cuda())
    q = torch.randn(s.n, 8, 64, dtype=torch.bfloat16, device="cuda")
    want, lse = s.pool.attention(s.seqs(), q, return_lse=True)
    fused = torch.zeros(s.n, 12 * 64, dtype=torch.bfloat16, device="cuda")
    part = fused[:, 64:64 * 9].view(s.n, 8, 64)
    part.copy_(q)
    out = torch.zeros(8, s.n, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    s.pool.attention(s.seqs(), part, out=out)
    assert torch.equal(out, want)
    s.pool.attention(s.seqs(), part, out=part)
    assert torch.equal(part, want) and (fused[:, :64] == 0).all() and (fused[:, 64 * 9:] == 0).all()


def test_decoding_with_all_three_in_a_captured_graph(pv):
    """Append, attention and read of a batch, captured once and replayed while lengths and data change in place; every replay against eager calls on a second pool."""
    lens, heads, hd = [30, 511, 0, 250], 2, 64
    a, b = (Setup(pv, [n + 24 for n in lens], [1] * 4, heads=heads, hd=hd, seed=9) for _ in range(2))
    for s in (a, b):
        s.prefix = list(lens)
        s.fill_prefix()
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda h: torch.randn(4, h, hd, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    k, v, q = draw(heads), draw(heads), draw(8)
    seqs = a.seqs()
    out, lse = torch.empty_like(q), torch.empty(4, 8, device="cuda")
    rk, rv = torch.empty_like(k), torch.empty_like(v)

    def step():
        a.pool.append(seqs, k, v)
        a.pool.attention(seqs, q, out=out, lse=lse)
        a.pool.read(seqs, 4, out=(rk, rv))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    eager = b.seqs()
    for i in range(12):
        graph.replay()
        torch.cuda.synchronize()
        b.pool.append(eager, k, v)
        w, wl = b.pool.attention(eager, q, return_lse=True)
        wk, wv = b.pool.read(eager, 4)
        assert torch.equal(out, w) and torch.equal(lse, wl) and torch.equal(rk, wk) and torch.equal(rv, wv), i
        assert torch.equal(a.pool.codes, b.pool.codes) and torch.equal(a.pool.scales, b.pool.scales)
        for x, h in ((k, heads), (v, heads), (q, 8)):
            x.copy_(draw(h))
        seqs.prefix_len.add_(1)
        eager.prefix_len.add_(1)
    torch.cuda.synchronize()


def test_two_streams_at_once(pv):
    sets = []
    for seed in (1, 2):
        s = Setup(pv, [1500, 700], [6, 6], heads=2, hd=128, seed=seed)
        s.fill_prefix()
        k, v = s.draw(s.n, "bf16", 0.5).cuda(), s.draw(s.n, "bf16").cuda()
        s.pool.append(s.seqs(), k, v)
        q = torch.randn(s.n, 8, 128, dtype=torch.bfloat16, device="cuda")
        sets.append((s, s.seqs(), q, s.pool.attention(s.seqs(), q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(8):
        for i, (s, seqs, q, _) in enumerate(sets):
            got[i].append(s.pool.attention(seqs, q, stream=streams[i]))
    torch.cuda.synchronize()
    for (_, _, _, want), outs in zip(sets, got):
        assert all(torch.equal(o, want) for o in outs)


@pytest.fixture()
def long_tables(monkeypatch):
    """Tables as of 20000 tokens, most of them of no page: what many rows over long contexts are worked through by, at sizes of a test."""
    monkeypatch.setattr(Setup, "room", 1250)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("prefix,rows,kvh,heads,pt", [([300], [1], 2, 8, 16), ([700], [4], 1, 5, 16), ([0, 40, 0, 511, 1000], [3, 0, 1, 9, 1], 2, 8, 16), ([5] * 70, [1] * 70, 1, 2, 16), ([300], [9], 2, 8, 16), ([255], [10], 1, 4, 64), ([1100], [33], 2, 4, 16), ([0], [17], 2, 8, 16), ([0], [130], 1, 4, 16), ([77], [65], 2, 6, 32),
                                                      ([513], [33], 1, 16, 16), ([0, 40, 0, 511, 1000], [30, 0, 11, 9, 41], 2, 8, 16), ([200, 0, 31], [1, 100, 40], 2, 8, 16), ([90], [5], 1, 70, 16)])
def test_many_rows_over_long_tables(pv, long_tables, prefix, rows, kvh, heads, pt, dtype, hd):
    test_attention(pv, prefix, rows, kvh, heads, pt, dtype, hd)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("prefix,rows", [([100], [48]), ([0], [9]), ([300, 0, 17], [64, 5, 20]), ([50], [70])])
def test_masks_over_long_tables(pv, long_tables, prefix, rows, dtype):
    test_attention_with_masks(pv, prefix, rows, dtype)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [10, 70])
def test_what_a_row_does_not_see_over_long_tables(pv, long_tables, bad, rows):
    test_what_a_row_does_not_see_has_no_influence(pv, bad, rows)


def test_missing_pages_and_strides_over_long_tables(pv, long_tables):
    test_pages_and_lengths_that_do_not_exist(pv)
    test_in_place_and_strided_queries(pv)


@pytest.mark.parametrize("rows", [1, 10, 40])
def test_scales_far_apart_for_any_number_of_rows(pv, monkeypatch, rows):
    """The case of the two rows, with as many as are worked through in other ways."""
    monkeypatch.setattr(Setup, "room", 1250)
    s = Setup(pv, [400], [rows], heads=1, hd=64)
    n = 400 + rows
    k, v = torch.from_numpy(s.r.normal(size=(n, 1, 64))).float() * 0.1, torch.from_numpy(s.r.normal(size=(n, 1, 64))).float()
    v[:200] *= 2.0 ** -20
    v[200:216] *= 2.0 ** 20
    k[200:216] = -k[0] * 100
    k[0], v[0] = 3.0, 1e-12
    s.pool.append(s.seqs([0, n], [0]), k.cuda(), v.cuda())
    s.ref.append([0, n], [0], s.tables, k.double().numpy(), v.double().numpy())
    q = (torch.ones(rows, 6, 64) * torch.linspace(1, 0.5, 6).view(1, 6, 1)).to(torch.bfloat16)
    for scale in (0.02, 0.07, -0.02):
        out, lse = s.pool.attention(s.seqs(), q.cuda(), scale=scale, return_lse=True)
        check_attention(s, q, out, lse, scale=scale)


def test_graphs_and_eager_calls_at_once(pv):
    """Calls of three kinds, captured apart, replayed on three streams while eager ones run on a fourth: nobody's workspace is another's."""
    calls = []
    for n, length, room in ((1, 2000, 0), (40, 2000, 1250), (9, 1500, 0)):
        s = Setup(pv, [length], [n], heads=2, hd=128, fill=0)
        s.pool.codes.random_(0, 120)
        s.pool.scales.fill_(120)
        s.room = room
        calls.append((s.pool, s.seqs(), torch.from_numpy(s.r.normal(size=(n, 8, 128))).to(torch.bfloat16).cuda()))
    want = [pool.attention(seqs, q, return_lse=True) for pool, seqs, q in calls]
    torch.cuda.synchronize()
    graphs = []
    for pool, seqs, q in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = pool.attention(seqs, q, return_lse=True)
        graphs.append((g, got))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for (g, got), x in zip(graphs, streams):
            got[0].zero_()
            x.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(x):
                g.replay()
        eager = [pool.attention(seqs, q, return_lse=True) for pool, seqs, q in calls]
        torch.cuda.synchronize()
        for (_, got), w, e in zip(graphs, want, eager):
            assert all(torch.equal(i, j) and torch.equal(k, j) for i, j, k in zip(got, w, e)) and torch.isfinite(w[0]).all()
