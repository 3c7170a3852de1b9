"""Attention over the 16-bit cache in tiles of 64 and 128 rows, whose keys and values go through LDS.

How a call is cut depends on its rows and on how far its tables reach, not on the lengths, which the host does not know: tables much longer than the sequences, without pages behind their ends, bring small calls to these tiles, and
tables of some thousand tokens to several chunks of keys.  Oracle and tolerances: tests/test_gpu_kv16.py."""
import numpy as np
import pytest
import torch

from test_gpu_kv16 import TYPES, Setup, check, dev, pv  # noqa: F401

pytestmark = pytest.mark.gpu


class Far(Setup):
    """Tables that reach for `reach` tokens."""

    def __init__(self, pv, case, hd, dtype, **more):  # noqa: F811
        prefix, rows, heads, self.q_heads, pt, reach = case
        super().__init__(pv, prefix, rows, heads=heads, hd=hd, pt=pt, dtype=dtype, **more)
        behind = np.full((len(rows), reach // pt - self.tables.shape[1]), -1, np.int32)
        behind[:, ::3] = self.pool.n_pages                                # neither is a page
        self.tables = np.concatenate([self.tables, behind], axis=1)

    def queries(self, size=1.0):
        return torch.from_numpy(self.r.normal(size=(self.n, self.q_heads, self.hd)) * size).to(self.dtype)


# prefix, rows, kv heads, query heads, page, reach: tiles of 64; of 128; several chunks, up to 16 and more
TILES = {
    "64, one tile": ([0], [9], 2, 8, 16, 1 << 17), "64, ends inside a step": ([70], [13], 3, 12, 16, 1 << 17), "64, ragged": ([5, 0, 130, 63], [12, 0, 3, 16], 2, 8, 16, 1 << 17),
    "64, an odd group": ([191], [8], 2, 14, 32, 1 << 17), "64, one head a kv head": ([64], [50], 4, 4, 64, 1 << 17),
    "128, one tile": ([0], [25], 2, 8, 16, 1 << 17), "128, ends inside a step": ([100], [57], 2, 8, 16, 1 << 17), "128, ragged": ([257, 0, 31, 9], [40, 0, 77, 60], 2, 8, 16, 1 << 17),
    "128, an odd group": ([64], [41], 1, 5, 128, 1 << 17), "128, one head a kv head": ([1], [200], 2, 2, 16, 1 << 17),
    "64, few chunks": ([900], [60], 4, 32, 16, 4096), "64, many chunks": ([1300], [25], 5, 20, 16, 1 << 14), "64, chunks of some": ([1500, 3, 300], [20, 9, 21], 4, 16, 32, 1 << 14),
    "128, few chunks": ([1000], [66], 4, 32, 16, 4096), "128, many chunks": ([1279], [41], 4, 16, 16, 1 << 14), "128, chunks of some": ([1700, 0, 255], [80, 70, 33], 4, 16, 16, 1 << 14),
}
tiles = pytest.mark.parametrize("case", list(TILES.values()), ids=list(TILES))


@tiles
@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 64)])
def test_attention(pv, case, dtype, hd):  # noqa: F811
    s = Far(pv, case, hd, dtype, tail_rows=1)
    s.fill_prefix()
    s.fill_rows()
    q = s.queries()
    out, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    s.pool.attention(s.seqs(), q.cuda(), out=out, lse=lse)
    assert (out[-1] == 7).all() and (lse[-1] == 7).all()
    check(s.ref, s.start, s.prefix, s.tables, q[:-1], out[:-1], lse[:-1])


@tiles
@pytest.mark.parametrize("dtype,hd,words", [("bf16", 128, 4), ("f16", 64, 1), ("bf16", 64, 60)])      # (60: more than there is room for beside the tiles)
def test_attention_with_masks(pv, case, dtype, hd, words):  # noqa: F811
    """Rows that see nothing of the block, or nothing at all; slots without a bit; words behind the rows."""
    s = Far(pv, case, hd, dtype)
    s.fill_prefix()
    s.fill_rows()
    m = s.r.integers(0, 2 ** 63, (s.n, words)).astype(np.int64)
    m[0], m[-1], m[s.n // 2] = 0, -1, 1
    whole = [sum(int(w) << (64 * i) for i, w in enumerate(row.view(np.uint64))) for row in m]
    q = s.queries()
    out, lse = s.pool.attention(s.seqs(), q.cuda(), mask=dev(m[:, 0] if words == 1 else m, torch.int64), return_lse=True)
    check(s.ref, s.start, s.prefix, s.tables, q, out, lse, masks=whole)


@pytest.mark.parametrize("name", ["64, ragged", "64, chunks of some", "64, many chunks", "128, ragged", "128, chunks of some", "128, few chunks"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 64)])
def test_pages_that_do_not_exist(pv, name, masked, dtype, hd):  # noqa: F811
    """The first page, some in the middle, the last of the sequence's; a sequence all of whose pages are none: its rows see nothing."""
    s = Far(pv, TILES[name], hd, dtype)
    s.fill_prefix()
    s.fill_rows()
    t, longest = s.tables.copy(), int(np.argmax(s.prefix))
    used = -(-(s.prefix[longest] + s.rows[longest]) // s.pool.page_tokens)
    t[longest, [0, used // 2, used // 2 + 1, used - 1]] = -1, s.pool.n_pages, -2 ** 31, 2 ** 31 - 1
    if len(s.rows) > 1:
        t[-1] = -1
    m = s.r.integers(0, 2 ** 63, (s.n, 2)).astype(np.int64)
    q = s.queries()
    out, lse = s.pool.attention(s.seqs(tables=t), q.cuda(), mask=dev(m, torch.int64) if masked else None, return_lse=True)
    check(s.ref, s.start, s.prefix, t, q, out, lse, masks=[int(a) | int(b) << 64 for a, b in m.view(np.uint64)] if masked else None)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("name", ["64, ends inside a step", "64, one head a kv head", "64, many chunks", "128, one tile", "128, ends inside a step", "128, many chunks"])
@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 64)])
def test_what_a_row_does_not_see_has_no_influence(pv, bad, name, dtype, hd):  # noqa: F811
    """A key or a value of the block that is not finite: rows that see it are not finite (of a value: in its feature), the others, bit for bit, what they are without it."""
    s = Far(pv, TILES[name], hd, dtype)
    s.fill_prefix()
    k, v, q, rows = s.draw(s.n, size=0.5), s.draw(s.n), s.queries().cuda(), s.n
    masks = [((1 << rows) - 1) & ~(1 << 5) if i % 3 else (1 << rows) - 1 for i in range(rows)]
    m = dev(np.array([[(x >> (64 * w)) & (2 ** 64 - 1) for w in range(-(-rows // 64))] for x in masks], dtype=np.uint64).view(np.int64), torch.int64)
    for mask in (None, m):
        sees = torch.tensor([(x >> 5) & 1 == 1 for x in masks] if mask is not None else [i >= 5 for i in range(rows)])
        s.pool.append(s.seqs(), k.cuda(), v.cuda())
        clean = s.pool.attention(s.seqs(), q, mask=mask).cpu()
        assert torch.isfinite(clean).all()
        for which in ("k", "v"):
            kk, vv = k.clone(), v.clone()
            (kk if which == "k" else vv)[5, 0, 9] = bad
            s.pool.append(s.seqs(), kk.cuda(), vv.cuda())
            out = s.pool.attention(s.seqs(), q, mask=mask).cpu()
            group = s.q_heads // s.heads
            assert torch.equal(out[~sees], clean[~sees]) and torch.equal(out[:, group:], clean[:, group:])       # (it is one kv head's)
            out, f = out[sees][:, :group], torch.arange(hd) == 9
            if which == "v":
                # (a weight is one number of the type, 0 where it is too small for one: infinity times 0 is NaN)
                assert torch.equal(out[..., ~f], clean[sees][:, :group][..., ~f])
                assert out[..., 9].isnan().all() if bad != bad else (out[..., 9].isnan() | (out[..., 9] == bad)).all()
            elif bad != bad:
                assert out.isnan().all()


@pytest.mark.parametrize("name", ["64, one tile", "64, many chunks", "128, ragged", "128, few chunks"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_that_rise_and_fall(pv, name, dtype):  # noqa: F811
    """Largest scores that come late, by steps less and more than what results are rescaled at, or first; none (a scale of 0); a negative scale."""
    for rise in (0.02, 0.2, -0.2):
        s = Far(pv, TILES[name], 64, dtype)
        total = [p + w for p, w in zip(s.prefix, s.rows)]
        place = np.concatenate([np.arange(n) for n in total])
        k, v = torch.zeros(len(place), s.heads, 64), s.draw(len(place))
        k[:, :, 0] = torch.from_numpy(np.clip(rise * (place - 100), -60, 60)).float()[:, None]
        s.put(np.concatenate([[0], np.cumsum(total)]).astype(np.int32), [0] * len(total), k.to(s.dtype), v)
        q = torch.zeros(s.n, s.q_heads, 64)
        q[..., 0] = torch.linspace(0.25, 1, s.q_heads)
        q = q.to(s.dtype)
        for scale in (1.0, -1.0, 0.0):
            out, lse = s.pool.attention(s.seqs(), q.cuda(), scale=scale, return_lse=True)
            check(s.ref, s.start, s.prefix, s.tables, q, out, lse, scale=scale)


@pytest.mark.parametrize("name", ["64, chunks of some", "128, chunks of some", "128, few chunks", "64, ragged"])
def test_graphs(pv, name):  # noqa: F811
    """Two graphs of the same shapes, replayed in turn after lengths and tables have changed, eager calls between them; causal and masked; a strided q with the result over it."""
    s = Far(pv, TILES[name], 128, "bf16")
    s.fill_prefix()
    s.fill_rows()
    fused = torch.randn(s.n, 2 * s.q_heads * 128, dtype=torch.bfloat16, device="cuda")
    q, rest = fused[:, :s.q_heads * 128].view(s.n, s.q_heads, 128), fused[:, s.q_heads * 128:].clone()
    m = dev(s.r.integers(0, 2 ** 63, (s.n, 2)), torch.int64)
    seqs, graphs, outs = s.seqs(), [], []
    for mask in (None, m):
        outs.append(torch.empty(s.n, s.q_heads, 128, dtype=torch.bfloat16, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.pool.attention(seqs, q, mask=mask, out=outs[-1])
    for i in range(4):
        seqs.prefix_len.copy_(dev([max(0, p - 70 * i) for p in s.prefix]))
        if i == 2:
            seqs.page_table[:, 0] = -1
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out, mask in zip(outs, (None, m)):
            fresh = s.pool.attention(seqs, q.contiguous(), mask=mask)
            assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(fresh)) and torch.equal(out.isnan(), fresh.isnan())
    want = s.pool.attention(seqs, q.contiguous())
    s.pool.attention(seqs, q, out=q)
    assert torch.equal(torch.nan_to_num(q), torch.nan_to_num(want)) and torch.equal(fused[:, s.q_heads * 128:], rest)
