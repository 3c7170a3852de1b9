"""The 8-bit cache's rules on the CPU: the test oracle's codes against torch's conversion, sizes, and what the entry points refuse (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2505_01572_amd import binding, operators


def test_oracle_codes_are_torchs():
    x = np.concatenate([ref.VALUES[:127], (ref.VALUES[:126] + ref.VALUES[1:127]) / 2, np.random.default_rng(0).uniform(0, 448, 4096), 2.0 ** -np.arange(20.0)])
    x = np.concatenate([x, -x])
    near = np.concatenate([x, np.nextafter(x.astype(np.float32), np.float32(np.inf)), np.nextafter(x.astype(np.float32), np.float32(-np.inf))]).astype(np.float32)
    near = near[np.abs(near) <= 448]
    want = torch.from_numpy(near).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(near), want)
    assert np.array_equal(ref.VALUES[ref.encode(ref.VALUES[:127])], ref.VALUES[:127])
    assert list(ref.encode([np.inf, np.nan])) == [0x7f, 0x7f]


def pool_arg(**kw):
    d = dict(codes=0x1000, scales=0x2000, n_pages=4, n_kv_heads=2, head_dim=64, page_tokens=16)
    d.update(kw)
    return binding.pv_kv8_pool(*d.values())


def seqs_arg(**kw):
    d = dict(row_start=0x1000, prefix_len=0x1000, page_table=0x1000, n_seq=1, n_rows=1, table_pages=4)
    d.update(kw)
    return binding.pv_kv8_seqs(*d.values())


def test_sizes():
    L = binding.lib()
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    for pages, heads, hd, pt in ((1, 1, 64, 16), (7, 3, 128, 16), (5, 8, 128, 256)):
        assert L.pv_kv8_bytes(ctypes.byref(pool_arg(codes=None, scales=None, n_pages=pages, n_kv_heads=heads, head_dim=hd, page_tokens=pt)), ctypes.byref(c), ctypes.byref(s)) == 0
        assert (c.value, s.value) == (pages * heads * 2 * pt * hd, pages * heads * 2 * pt // 16)
    b = ctypes.c_size_t(1)
    assert L.pv_kv8_attention_bytes(ctypes.byref(pool_arg()), ctypes.byref(seqs_arg(n_seq=0)), 2, ctypes.byref(b)) == 0 and b.value == 0


BAD_POOLS = [(dict(codes=None), -1), (dict(scales=None), -1), (dict(head_dim=32), -1), (dict(head_dim=96), -1), (dict(n_pages=0), -3), (dict(n_pages=1 << 26), -3), (dict(n_kv_heads=0), -3),
             (dict(page_tokens=8), -1), (dict(page_tokens=48), -1), (dict(page_tokens=1 << 17), -1), (dict(codes=0x1008), -1), (dict(scales=0x2001), -1),
             (dict(n_kv_heads=512, head_dim=64, page_tokens=1 << 16), -3)]
BAD_SEQS = [(dict(row_start=None), -1), (dict(prefix_len=None), -1), (dict(page_table=None), -1), (dict(n_seq=-1), -3), (dict(n_rows=-1), -3), (dict(table_pages=-1), -3),
            (dict(n_seq=(1 << 20) + 1), -3), (dict(n_rows=(1 << 24) + 1), -3)]


@pytest.mark.parametrize("pool,seqs,status", [(p, {}, st) for p, st in BAD_POOLS] + [({}, q, st) for q, st in BAD_SEQS])
def test_pools_and_sequences_are_checked(pool, seqs, status):
    L, p, q = binding.lib(), pool_arg(**pool), seqs_arg(**seqs)
    rows = (0x1000, 128, 64)
    assert L.pv_kv8_append(ctypes.byref(p), ctypes.byref(q), *rows, *rows, 1, None) == status
    assert L.pv_kv8_read(ctypes.byref(p), ctypes.byref(q), *rows, *rows, 1, None) == status
    assert L.pv_kv8_attention(ctypes.byref(p), ctypes.byref(q), *rows, 2, None, 1.0, *rows, None, 1, None, 0, None) == status
    assert L.pv_last_error()


def test_rows_are_checked():
    L, p, q = binding.lib(), pool_arg(), seqs_arg()
    good = (0x1000, 128, 64)
    for bad in ((None, 128, 64), (0x1008, 128, 64), (0x1000, 100, 64), (0x1000, 128, 60), (0x1000, -128, 64)):
        assert L.pv_kv8_append(ctypes.byref(p), ctypes.byref(q), *bad, *good, 1, None) == -1
        assert L.pv_kv8_append(ctypes.byref(p), ctypes.byref(q), *good, *bad, 1, None) == -1
        assert L.pv_kv8_read(ctypes.byref(p), ctypes.byref(q), *good, *bad, 1, None) == -1
        assert L.pv_kv8_attention(ctypes.byref(p), ctypes.byref(q), *bad, 2, None, 1.0, *good, None, 1, None, 0, None) == -1
        assert L.pv_kv8_attention(ctypes.byref(p), ctypes.byref(q), *good, 2, None, 1.0, *bad, None, 1, None, 0, None) == -1
    assert L.pv_kv8_append(ctypes.byref(p), ctypes.byref(q), *good, *good, 3, None) == -1


def test_attention_arguments_are_checked():
    L, p = binding.lib(), pool_arg()

    def call(q=None, heads=2, scale=1.0, lse=None, mask=None, dtype=1, ws=None, nbytes=0, pool=p):
        rows = (0x1000, 1 << 20, 64)
        return L.pv_kv8_attention(ctypes.byref(pool), ctypes.byref(q or seqs_arg()), *rows, heads, mask, scale, *rows, lse, dtype, ws, nbytes, None)
    assert call(heads=3) == call(heads=0) == call(heads=-2) == -1
    assert call(scale=float("inf")) == call(scale=float("nan")) == -1
    assert call(dtype=0) == call(dtype=5) == -1
    assert call(lse=0x1002) == call(mask=0x1004) == -1
    assert call(seqs_arg(n_rows=1 << 20), heads=32) == -3
    assert call(seqs_arg(table_pages=(1 << 26) + 1)) == -3
    long = seqs_arg(table_pages=4096)
    need = ctypes.c_size_t()
    assert L.pv_kv8_attention_bytes(ctypes.byref(p), ctypes.byref(long), 2, ctypes.byref(need)) == 0 and need.value > 0
    assert call(long) == call(long, ws=0x1000, nbytes=need.value - 1) == -5
    assert call(long, ws=0x1008, nbytes=need.value) == -1


def test_empty_calls_do_nothing():
    L, p, rows = binding.lib(), pool_arg(), (None, 0, 0)
    for q in (seqs_arg(n_rows=0), seqs_arg(n_seq=0, row_start=None, prefix_len=None, page_table=None)):
        assert L.pv_kv8_append(ctypes.byref(p), ctypes.byref(q), *rows, *rows, 1, None) == 0
        assert L.pv_kv8_read(ctypes.byref(p), ctypes.byref(q), *rows, *rows, 1, None) == 0
        assert L.pv_kv8_attention(ctypes.byref(p), ctypes.byref(q), *rows, 2, None, 1.0, *rows, None, 1, None, 0, None) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(binding.PVError):
        operators.KV8Seqs(i(2), i(1), i(1, 4))
    with pytest.raises(binding.PVError):
        operators.KV8Pool(4, 2, 64, codes=torch.zeros(4, 2, 2, 1024, dtype=torch.uint8), scales=torch.zeros(4, 2, 1, 2, dtype=torch.uint8))
    with pytest.raises(binding.PVError):
        operators.KV8Pool(4, 2, 80)
