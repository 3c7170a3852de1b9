"""Operators on the caller's own tensors (include/pipeverify.h, "operators around a key/value cache in 8 bits" and pv_token_logprobs).

    pool = pv.KV8Pool(n_pages, n_kv_heads, head_dim)                  # pages shared by all sequences (one pool a layer)
    seqs = pv.KV8Seqs(row_start, prefix_len, page_table)              # int32 tensors on the device, read when the kernels run
    pool.append(seqs, k, v)                                           # quantise the rows' keys and values into the pages
    out = pool.attention(seqs, q)                                     # every row over its sequence's prefix and its block
    got = pv.token_logprobs(logits, tokens, top=5)                    # log probabilities, entropy, alternatives

Argument marshalling only; work is enqueued on `stream` (default: the current stream of the pool's device) and not waited for.  A tensor made on another stream
is the caller's to order, as everywhere in torch.
"""
import ctypes
import math

import torch

from .binding import PVError, TokenLogprobs, _check, lib, pv_kv8_pool, pv_kv8_seqs

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _need(ok, where, what):
    if not ok:
        raise PVError(-1, where, what)


def _on(t, device, where, name):
    _need(isinstance(t, torch.Tensor) and t.device == device, where, f"{name} is not a tensor on {device}")


class _Stream:
    """Makes device and stream current, so that what torch allocates belongs to the stream the kernels run on."""

    def __init__(self, device, stream):
        self.stream = torch.cuda.current_stream(device) if stream is None else stream
        self.ctx = torch.cuda.stream(self.stream)

    def __enter__(self):
        self.ctx.__enter__()
        return ctypes.c_void_p(self.stream.cuda_stream)

    def __exit__(self, *a):
        return self.ctx.__exit__(*a)


class KV8Seqs:
    """A ragged batch: sequence s has rows row_start[s] .. row_start[s + 1] - 1 of a call's rows, at positions prefix_len[s] ... of its tokens, and
    page_table[s, i] is the physical page of its tokens i * page_tokens ....  Contiguous int32 tensors on one device, [n + 1], [n] and [n, pages]; what they
    hold is read when a call's kernels run, so they may be changed in place between replays of a captured graph."""

    def __init__(self, row_start, prefix_len, page_table):
        where = "KV8Seqs"
        for name, t, dims in (("row_start", row_start, 1), ("prefix_len", prefix_len, 1), ("page_table", page_table, 2)):
            _need(isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.dim() == dims and t.is_contiguous(), where, f"{name} must be a contiguous int32 tensor of {dims} dimension(s)")
            _need(t.is_cuda and t.device == prefix_len.device, where, f"{name} must be on the GPU, all three on one device")
        n = prefix_len.shape[0]
        _need(row_start.shape[0] == n + 1 and page_table.shape[0] == n, where, f"{n} sequences: row_start must have {n + 1} entries, page_table {n} rows")
        self.row_start, self.prefix_len, self.page_table, self.device = row_start, prefix_len, page_table, prefix_len.device

    def _arg(self, n_rows):
        return pv_kv8_seqs(self.row_start.data_ptr(), self.prefix_len.data_ptr(), self.page_table.data_ptr(), self.prefix_len.shape[0], n_rows, self.page_table.shape[1])


class KV8Pool:
    """Pages of an 8-bit key/value cache.  codes, scales: the two arrays (uint8, [n_pages, n_kv_heads, 2, page_tokens * head_dim] and
    [n_pages, n_kv_heads, page_tokens / 16, 2]); made here unless given."""

    def __init__(self, n_pages, n_kv_heads, head_dim, page_tokens=16, codes=None, scales=None, device="cuda:0"):
        where = "KV8Pool"
        self.L = lib()
        nc, ns = ctypes.c_size_t(), ctypes.c_size_t()
        _check(self.L.pv_kv8_bytes(ctypes.byref(pv_kv8_pool(None, None, n_pages, n_kv_heads, head_dim, page_tokens)), ctypes.byref(nc), ctypes.byref(ns)), "pv_kv8_bytes")
        self.n_pages, self.n_kv_heads, self.head_dim, self.page_tokens = n_pages, n_kv_heads, head_dim, page_tokens
        shapes = ((n_pages, n_kv_heads, 2, page_tokens * head_dim), (n_pages, n_kv_heads, page_tokens // 16, 2))
        given = codes if codes is not None else scales
        self.device = given.device if given is not None else torch.device(device)
        self.codes = torch.empty(shapes[0], dtype=torch.uint8, device=self.device) if codes is None else codes
        self.scales = torch.empty(shapes[1], dtype=torch.uint8, device=self.device) if scales is None else scales
        self.device = self.codes.device
        for name, t, shape in (("codes", self.codes, shapes[0]), ("scales", self.scales, shapes[1])):
            _on(t, self.device, where, name)
            _need(t.is_cuda and t.dtype == torch.uint8 and tuple(t.shape) == shape and t.is_contiguous(), where, f"{name} must be a contiguous uint8 tensor {shape} on the GPU")

    def _arg(self):
        return ctypes.byref(pv_kv8_pool(self.codes.data_ptr(), self.scales.data_ptr(), self.n_pages, self.n_kv_heads, self.head_dim, self.page_tokens))

    def _seqs(self, seqs, where, n_rows):
        _need(isinstance(seqs, KV8Seqs) and seqs.device == self.device, where, f"seqs must be a KV8Seqs on {self.device}")
        return ctypes.byref(seqs._arg(n_rows))

    def _rows(self, t, where, name, heads, dtypes, rows=None, like=None):
        """Address and strides of rows [n, heads, head_dim], features next to each other."""
        _on(t, self.device, where, name)
        _need(t.dtype in dtypes and t.dim() == 3 and t.shape[1] == heads and t.shape[2] == self.head_dim, where, f"{name} must be [rows, {heads}, {self.head_dim}] of {dtypes}, got {tuple(t.shape)} of {t.dtype}")
        _need(rows is None or t.shape[0] == rows, where, f"{name} must have {rows} rows")
        _need(like is None or t.dtype == like.dtype, where, f"{name} must be {like.dtype if like is not None else None}")
        _need(t.stride(2) == 1 or t.numel() == 0, where, f"{name}: the features of a head must lie next to each other")
        return t.data_ptr(), t.stride(0), t.stride(1)

    def append(self, seqs, k, v, stream=None):
        """Quantise k, v [rows, n_kv_heads, head_dim] (float32, bfloat16 or float16) into the pages of their sequences."""
        where = "KV8Pool.append"
        ka = self._rows(k, where, "k", self.n_kv_heads, tuple(_DTYPES))
        va = self._rows(v, where, "v", self.n_kv_heads, tuple(_DTYPES), k.shape[0], k)
        sa = self._seqs(seqs, where, k.shape[0])
        with _Stream(self.device, stream) as s:
            _check(self.L.pv_kv8_append(self._arg(), sa, *ka, *va, _DTYPES[k.dtype], s), "pv_kv8_append")

    def read(self, seqs, rows, dtype=torch.bfloat16, out=None, stream=None):
        """The tokens at the rows' positions, dequantised: (k, v), each [rows, n_kv_heads, head_dim].  out: the pair to write to (rows of no
        sequence are left as they are); made here otherwise."""
        where = "KV8Pool.read"
        with _Stream(self.device, stream) as s:
            if out is None:
                _need(dtype in _DTYPES, where, f"dtype must be one of {tuple(_DTYPES)}")
                out = tuple(torch.empty(rows, self.n_kv_heads, self.head_dim, dtype=dtype, device=self.device) for _ in range(2))
            k, v = out
            ka = self._rows(k, where, "k", self.n_kv_heads, tuple(_DTYPES), rows)
            va = self._rows(v, where, "v", self.n_kv_heads, tuple(_DTYPES), rows, k)
            _check(self.L.pv_kv8_read(self._arg(), self._seqs(seqs, where, rows), *ka, *va, _DTYPES[k.dtype], s), "pv_kv8_read")
        return k, v

    def attention(self, seqs, q, scale=None, mask=None, out=None, return_lse=False, lse=None, stream=None):
        """softmax(scale q K^T) V of every row of q [rows, n_q_heads, head_dim] (bfloat16 or float16) over its sequence's tokens; scale: 1 / sqrt(head_dim) unless
        given.  Without a mask a row sees the tokens up to its own position.  mask: int64 or uint64 [rows], bit t: the row sees token prefix_len + t
        (a draft tree: its ancestors and itself); all tokens before prefix_len are seen.  Returns out, or (out, lse) with lse float32 [rows, n_q_heads]."""
        where = "KV8Pool.attention"
        _need(isinstance(q, torch.Tensor) and q.dim() == 3, where, "q must be [rows, heads, head_dim]")
        n, heads = q.shape[:2]
        scale = 1 / math.sqrt(self.head_dim) if scale is None else float(scale)
        half = (torch.bfloat16, torch.float16)
        qa = self._rows(q, where, "q", heads, half)
        if mask is not None:
            _on(mask, self.device, where, "mask")
            _need(mask.dtype in (torch.int64, torch.uint64) and tuple(mask.shape) == (n,) and mask.is_contiguous(), where, f"mask must be a contiguous int64 tensor [{n}]")
        pa, sa, need = self._arg(), self._seqs(seqs, where, n), ctypes.c_size_t()
        _check(self.L.pv_kv8_attention_bytes(pa, sa, heads, ctypes.byref(need)), "pv_kv8_attention_bytes")
        with _Stream(self.device, stream) as s:
            out = torch.empty(n, heads, self.head_dim, dtype=q.dtype, device=self.device) if out is None else out
            oa = self._rows(out, where, "out", heads, half, n, q)
            if lse is None and return_lse:
                lse = torch.empty(n, heads, dtype=torch.float32, device=self.device)
            if lse is not None:
                _on(lse, self.device, where, "lse")
                _need(lse.dtype == torch.float32 and tuple(lse.shape) == (n, heads) and lse.is_contiguous(), where, f"lse must be a contiguous float32 tensor [{n}, {heads}]")
            ws = torch.empty(need.value, dtype=torch.uint8, device=self.device) if need.value else None
            _check(self.L.pv_kv8_attention(pa, sa, *qa, heads, None if mask is None else mask.data_ptr(), scale, *oa, None if lse is None else lse.data_ptr(),
                                           _DTYPES[q.dtype], None if ws is None else ws.data_ptr(), need.value, s), "pv_kv8_attention")
        return (out, lse) if lse is not None else out


def token_logprobs(logits, tokens=None, top=0, stream=None):
    """Log probabilities under each row of logits [rows, vocab] (float32, bfloat16 or float16): of tokens (int32 [rows, n] or [rows]), and of the `top` <= 32 most
    probable ones (equal ones: the lower id first), with the row's entropy and log-sum-exp.  float32, in nats; a NaN logit counts as -infinity."""
    where = "token_logprobs"
    _need(isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2 and logits.dtype in _DTYPES, where, f"logits must be [rows, vocab] of {tuple(_DTYPES)} on the GPU")
    rows, vocab = logits.shape
    _need(logits.stride(1) == 1 or vocab <= 1 or rows == 0, where, "the logits of a row must lie next to each other")
    d = logits.device
    if tokens is not None:
        _on(tokens, d, where, "tokens")
        _need(tokens.dtype == torch.int32 and tokens.dim() in (1, 2) and tokens.shape[0] == rows and tokens.is_contiguous(), where, f"tokens must be a contiguous int32 tensor [{rows}] or [{rows}, n]")
    n = 0 if tokens is None else tokens.numel() // max(1, rows)
    L, need = lib(), ctypes.c_size_t()
    _check(L.pv_token_logprobs_bytes(rows, vocab, top, ctypes.byref(need)), "pv_token_logprobs_bytes")
    with _Stream(d, stream) as s:
        f = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=d)  # noqa: E731
        got = TokenLogprobs(f(*(tokens.shape if tokens is not None else (rows, 0))), f(rows), f(rows), torch.empty(rows, top, dtype=torch.int32, device=d), f(rows, top))
        ws = torch.empty(need.value, dtype=torch.uint8, device=d) if need.value else None
        p = lambda t: None if t is None or t.numel() == 0 else t.data_ptr()  # noqa: E731
        _check(L.pv_token_logprobs(logits.data_ptr(), logits.stride(0), _DTYPES[logits.dtype], rows, vocab, p(tokens), n, p(got.logprobs), p(got.entropy), p(got.lse),
                                   top, p(got.top_ids), p(got.top_logprobs), p(ws), need.value, s), "pv_token_logprobs")
    return got
