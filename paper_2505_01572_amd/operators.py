"""Operators on the caller's own tensors (include/pipeverify.h, "operators around a key/value cache in 8 bits" and pv_token_logprobs).

    pool = pv.KV8Pool(n_pages, n_kv_heads, head_dim)                  # pages shared by all sequences (one pool a layer)
    seqs = pv.KV8Seqs(row_start, prefix_len, page_table)              # int32 tensors on the device, read when the kernels run
    pool.append(seqs, k, v)                                           # quantise the rows' keys and values into the pages
    out = pool.attention(seqs, q)                                     # every row over its sequence's prefix and its block
    got = pv.token_logprobs(logits, tokens, top=5)                    # log probabilities, entropy, alternatives

Argument marshalling only; work is enqueued on `stream` (default: the current stream of the pool's device) and not waited for.  A tensor made on another stream
is the caller's to order, as everywhere in torch.  There are no gradients: tensors that require one are refused, unless gradients are switched off (torch.no_grad()).
"""
import ctypes

import torch

from .binding import PVError, TokenLogprobs, _check, lib, pv_kv8_pool, pv_kv8_seqs

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else lambda i: torch.cuda.current_stream(i).cuda_stream

# A call's Python takes about as long as its kernels on small batches, so what every call passes through formats no message and makes no object that it does not need.


def _refuse(where, what):
    raise PVError(-1, where, what)


class _Elsewhere:
    """Makes device and stream current, so that what torch allocates belongs to the stream the kernels run on."""

    def __init__(self, device, stream):
        if stream is not None and stream.device != device:
            _refuse("stream", f"a stream of {stream.device} given for tensors on {device}")
        self.device, self.stream = torch.cuda.device(device), torch.cuda.stream(stream) if stream is not None else None

    def __enter__(self):
        self.device.__enter__()
        if self.stream is not None:
            self.stream.__enter__()

    def __exit__(self, *a):
        if self.stream is not None:
            self.stream.__exit__(*a)
        self.device.__exit__(*a)


def _no_gradient(where, name, t):
    """There is no backward pass: a result without a history where torch would give one would be a gradient lost in silence."""
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(where, f"{name} requires a gradient, and this operator has none: call it under torch.no_grad(), or with {name}.detach()")


def _elsewhere(index, stream):
    return stream is not None or torch.cuda.current_device() != index


class KV8Seqs:
    """A ragged batch: sequence s has rows row_start[s] .. row_start[s + 1] - 1 of a call's rows, at positions prefix_len[s] ... of its tokens, and
    page_table[s, i] is the physical page of its tokens i * page_tokens ....  Contiguous int32 tensors on one device, [n + 1], [n] and [n, pages]; what they
    hold is read when a call's kernels run, so they may be changed in place between replays of a captured graph."""

    def __init__(self, row_start, prefix_len, page_table):
        where = "KV8Seqs"
        for name, t, dims in (("row_start", row_start, 1), ("prefix_len", prefix_len, 1), ("page_table", page_table, 2)):
            if not (isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.dim() == dims and t.is_contiguous()):
                _refuse(where, f"{name} must be a contiguous int32 tensor of {dims} dimension(s)")
            if not (t.is_cuda and t.device == row_start.device):
                _refuse(where, f"{name} must be on the GPU, all three on one device")
        n = prefix_len.shape[0]
        if row_start.shape[0] != n + 1 or page_table.shape[0] != n:
            _refuse(where, f"{n} sequences: row_start must have {n + 1} entries, page_table {n} rows")
        self.row_start, self.prefix_len, self.page_table, self.device = row_start, prefix_len, page_table, prefix_len.device
        self._fields = (row_start.data_ptr(), prefix_len.data_ptr(), page_table.data_ptr(), n)
        self._args = {}                                    # a call's rows -> the struct for it

    def _arg(self, n_rows):
        a = self._args.get(n_rows)
        if a is None:
            if len(self._args) > 256:
                self._args.clear()
            a = self._args[n_rows] = pv_kv8_seqs(*self._fields, n_rows, self.page_table.shape[1])
        return a


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
        at = given.device if given is not None else torch.device(device)
        self.codes = torch.empty(shapes[0], dtype=torch.uint8, device=at) if codes is None else codes
        self.scales = torch.empty(shapes[1], dtype=torch.uint8, device=at) if scales is None else scales
        self.device = self.codes.device
        for name, t, shape in (("codes", self.codes, shapes[0]), ("scales", self.scales, shapes[1])):
            if not (t.is_cuda and t.device == self.device and t.dtype == torch.uint8 and tuple(t.shape) == shape and t.is_contiguous()):
                _refuse(where, f"{name} must be a contiguous uint8 tensor {shape} on the GPU, both on one device")
        self._index = self.device.index
        self._arg = pv_kv8_pool(self.codes.data_ptr(), self.scales.data_ptr(), n_pages, n_kv_heads, head_dim, page_tokens)
        self._need = {}                                    # (sequences, rows, heads, table's pages) -> bytes of attention's workspace

    def _rows(self, t, where, name, heads, dtypes):
        """Rows [n, heads, head_dim], features next to each other: address and strides."""
        if not isinstance(t, torch.Tensor) or t.device != self.device:
            _refuse(where, f"{name} is not a tensor on {self.device}")
        shape, stride = t.shape, t.stride()
        if t.dtype not in dtypes or len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim:
            _refuse(where, f"{name} must be [rows, {heads}, {self.head_dim}] of {tuple(dtypes)}, got {tuple(shape)} of {t.dtype}")
        if stride[2] != 1:
            _refuse(where, f"{name}: the features of a head must lie next to each other")
        if t.requires_grad:
            _no_gradient(where, name, t)
        return t.data_ptr(), stride[0], stride[1]

    def _seqs(self, seqs, where, n_rows):
        if not isinstance(seqs, KV8Seqs) or seqs.device != self.device:
            _refuse(where, f"seqs must be a KV8Seqs on {self.device}")
        return seqs._arg(n_rows)

    def append(self, seqs, k, v, stream=None):
        """Quantise k, v [rows, n_kv_heads, head_dim] (float32, bfloat16 or float16) into the pages of their sequences."""
        where = "KV8Pool.append"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.append(seqs, k, v)
        kp, kr, kh = self._rows(k, where, "k", self.n_kv_heads, _DTYPES)
        vp, vr, vh = self._rows(v, where, "v", self.n_kv_heads, _DTYPES)
        n = k.shape[0]
        if v.shape[0] != n or v.dtype != k.dtype:
            _refuse(where, "k and v must have the same rows and type")
        rc = self.L.pv_kv8_append(self._arg, self._seqs(seqs, where, n), kp, kr, kh, vp, vr, vh, _DTYPES[k.dtype], _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv8_append")

    def read(self, seqs, rows, dtype=torch.bfloat16, out=None, stream=None):
        """The tokens at the rows' positions, dequantised: (k, v), each [rows, n_kv_heads, head_dim].  out: the pair to write to (rows of no
        sequence are left as they are); made here otherwise."""
        where = "KV8Pool.read"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.read(seqs, rows, dtype, out)
        if out is None:
            if dtype not in _DTYPES:
                _refuse(where, f"dtype must be one of {tuple(_DTYPES)}")
            out = torch.empty((2, rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device).unbind(0)
        k, v = out
        kp, kr, kh = self._rows(k, where, "k", self.n_kv_heads, _DTYPES)
        vp, vr, vh = self._rows(v, where, "v", self.n_kv_heads, _DTYPES)
        if k.shape[0] != rows or v.shape[0] != rows or v.dtype != k.dtype:
            _refuse(where, f"k and v must have {rows} rows and the same type")
        rc = self.L.pv_kv8_read(self._arg, self._seqs(seqs, where, rows), kp, kr, kh, vp, vr, vh, _DTYPES[k.dtype], _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv8_read")
        return k, v

    def attention(self, seqs, q, scale=None, mask=None, out=None, return_lse=False, lse=None, stream=None):
        """softmax(scale q K^T) V of every row of q [rows, n_q_heads, head_dim] (bfloat16 or float16) over its sequence's tokens; scale: 1 / sqrt(head_dim) unless
        given.  Without a mask a row sees the tokens up to its own position.  mask: int64 or uint64 [rows], bit t: the row sees token prefix_len + t
        (a draft tree: its ancestors and itself), t less than 64 and than the sequence's rows in the call; all tokens before prefix_len are seen.  Returns out, or (out, lse) with lse float32 [rows, n_q_heads]."""
        where = "KV8Pool.attention"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.attention(seqs, q, scale, mask, out, return_lse, lse)
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            _refuse(where, "q must be [rows, heads, head_dim]")
        n, heads, _ = q.shape
        qp, qr, qh = self._rows(q, where, "q", heads, _HALF)
        sa, mp = self._seqs(seqs, where, n), None
        if mask is not None:
            if not (isinstance(mask, torch.Tensor) and mask.device == self.device and mask.dtype in (torch.int64, torch.uint64) and mask.shape == (n,) and mask.is_contiguous()):
                _refuse(where, f"mask must be a contiguous int64 tensor [{n}] on {self.device}")
            mp = mask.data_ptr()
        key = (sa.n_seq, n, heads, sa.table_pages)
        need = self._need.get(key)
        if need is None:
            b = ctypes.c_size_t()
            _check(self.L.pv_kv8_attention_bytes(self._arg, sa, heads, ctypes.byref(b)), "pv_kv8_attention_bytes")
            if len(self._need) > 256:
                self._need.clear()
            need = self._need[key] = b.value
        if out is None:
            out = q.new_empty((n, heads, self.head_dim))
            op, orow, oh = out.data_ptr(), heads * self.head_dim, self.head_dim
        else:
            op, orow, oh = self._rows(out, where, "out", heads, _HALF)
            if out.shape[0] != n or out.dtype != q.dtype:
                _refuse(where, f"out must have {n} rows of {q.dtype}")
        if lse is not None:
            if not (isinstance(lse, torch.Tensor) and lse.device == self.device and lse.dtype == torch.float32 and lse.shape == (n, heads) and lse.is_contiguous()):
                _refuse(where, f"lse must be a contiguous float32 tensor [{n}, {heads}] on {self.device}")
            if lse.requires_grad:
                _no_gradient(where, "lse", lse)
        elif return_lse:
            lse = q.new_empty((n, heads), dtype=torch.float32)
        ws = q.new_empty(need, dtype=torch.uint8) if need else None
        rc = self.L.pv_kv8_attention(self._arg, sa, qp, qr, qh, heads, mp, self.head_dim ** -0.5 if scale is None else scale, op, orow, oh, None if lse is None else lse.data_ptr(),
                                     _HALF[q.dtype], None if ws is None else ws.data_ptr(), need, _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv8_attention")
        return out if lse is None else (out, lse)


_logprobs_need = {}                                        # (rows, vocab, top) -> bytes of workspace


def token_logprobs(logits, tokens=None, top=0, stream=None):
    """Log probabilities under each row of logits [rows, vocab] (float32, bfloat16 or float16): of tokens (int32 [rows, n] or [rows]), and of the `top` <= 32 most
    probable ones (equal ones: the lower id first), with the row's entropy and log-sum-exp.  float32, in nats; a NaN logit counts as -infinity."""
    where = "token_logprobs"
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2 and logits.dtype in _DTYPES):
        _refuse(where, f"logits must be [rows, vocab] of {tuple(_DTYPES)} on the GPU")
    if logits.requires_grad:
        _no_gradient(where, "logits", logits)
    index = logits.device.index
    if _elsewhere(index, stream):
        with _Elsewhere(logits.device, stream):
            return token_logprobs(logits, tokens, top)
    rows, vocab = logits.shape
    row_stride, one = logits.stride()
    if one != 1 and vocab > 1 and rows > 0:
        _refuse(where, "the logits of a row must lie next to each other")
    n, shape, tp = 0, (rows, 0), None
    if tokens is not None:
        if not (isinstance(tokens, torch.Tensor) and tokens.device == logits.device and tokens.dtype == torch.int32 and tokens.dim() in (1, 2) and tokens.shape[0] == rows and tokens.is_contiguous()):
            _refuse(where, f"tokens must be a contiguous int32 tensor [{rows}] or [{rows}, n] on {logits.device}")
        shape, tp = tokens.shape, tokens.data_ptr()
        n = 1 if len(shape) == 1 else shape[1]
    L, key = lib(), (rows, vocab, top)
    need = _logprobs_need.get(key)
    if need is None:
        b = ctypes.c_size_t()
        _check(L.pv_token_logprobs_bytes(rows, vocab, top, ctypes.byref(b)), "pv_token_logprobs_bytes")
        if len(_logprobs_need) > 256:
            _logprobs_need.clear()
        need = _logprobs_need[key] = b.value
    if n == 1:                                             # (one allocation for all three)
        lp, entropy, lse = logits.new_empty((3, rows), dtype=torch.float32).unbind(0)
        if len(shape) == 2:
            lp = lp.view(shape)
    else:
        lp = logits.new_empty(shape, dtype=torch.float32)
        entropy, lse = logits.new_empty((2, rows), dtype=torch.float32).unbind(0)
    ids, best = logits.new_empty((rows, top), dtype=torch.int32), logits.new_empty((rows, top), dtype=torch.float32)
    ws = logits.new_empty(need, dtype=torch.uint8) if need else None
    rc = L.pv_token_logprobs(logits.data_ptr(), row_stride, _DTYPES[logits.dtype], rows, vocab, tp, n, lp.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                             top, ids.data_ptr(), best.data_ptr(), None if ws is None else ws.data_ptr(), need, _raw_stream(index))
    if rc:
        _check(rc, "pv_token_logprobs")
    return TokenLogprobs(lp, entropy, lse, ids, best)
