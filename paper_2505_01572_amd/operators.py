"""Operators on the caller's own tensors (include/pipeverify.h, "operators around a key/value cache in 8 bits", pv_token_logprobs, "operators around a key/value cache in 16 bits, and drafts verified by sampling").

    pool = pv.KV8Pool(n_pages, n_kv_heads, head_dim)                  # pages shared by all sequences (one pool a layer)
    seqs = pv.KV8Seqs(row_start, prefix_len, page_table)              # int32 tensors on the device, read when the kernels run
    pool.append(seqs, k, v)                                           # quantise the rows' keys and values into the pages
    out = pool.attention(seqs, q)                                     # every row over its sequence's prefix and its block
    got = pv.token_logprobs(logits, tokens, top=5)                    # log probabilities, entropy, alternatives

    pool = pv.KV16Pool(n_pages, n_kv_heads, head_dim)                 # the same in bfloat16 or float16
    rotary = pv.Rotary(head_dim, base=500000.0)
    q = pool.append(seqs, k, v, rotary=rotary, q=q)                   # keys rotated on their way into the pages, and the queries of the same rows
    out = pool.attention(seqs, q, mask=mask)                          # a draft tree of any number of nodes
    got = pv.verify_drafts(row_start, logits, tokens, u, parent=parent, temperature=0.7)      # drafts taken by the target's probabilities, the token that follows
    pool.keep(seqs, got.path, got.accepted)                           # the accepted path behind the prefix

Argument marshalling only; work is enqueued on `stream` (default: the current stream of the pool's device) and not waited for.  A tensor made on another stream
is the caller's to order, as everywhere in torch.  There are no gradients: tensors that require one are refused, unless gradients are switched off (torch.no_grad()), and so are tensors that
carry a tangent of forward mode.
"""
import ctypes
import math

import torch
from torch.autograd import forward_ad

from .binding import DraftVerdict, PVError, TokenLogprobs, _check, lib, pv_kv16_pool, pv_kv8_pool, pv_kv8_seqs, pv_rotary

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


def _asks(t):
    """Whether a tensor may ask for a derivative (the level of forward mode, -1 outside of it, is looked at first: asking a tensor for its tangent takes some 0.3 us)."""
    return t.requires_grad or forward_ad._current_level >= 0


def _no_gradient(where, name, t):
    """There is no backward pass, and no forward-mode one: a result without a history or a tangent where torch would give one would be a gradient lost in silence."""
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(where, f"{name} requires a gradient, and this operator has none: call it under torch.no_grad(), or with {name}.detach()")
    if forward_ad.unpack_dual(t).tangent is not None:
        _refuse(where, f"{name} carries a forward-mode gradient, and this operator has none: call it with the primal of {name}")


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
        if _asks(t):
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
            if _asks(lse):
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
    if _asks(logits):
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


KVSeqs = KV8Seqs                                           # the batches of both pools


class Rotary:
    """Rotary positions: pair i of a head's first rotary_dim features turns by position * frequency i, frequency i = base^(-2i / rotary_dim).  interleaved: pairs (2i, 2i + 1) instead of
    (i, i + rotary_dim / 2).  scaling: a dict for contexts longer than the trained one, of a "kind" and its numbers:
      linear  factor                              every frequency divided by factor
      base    factor                              base times factor^(rotary_dim / (rotary_dim - 2)): the fastest pair stays, the slowest is divided by factor
      turns   factor, original, low, high         divided where the pair makes up to `low` turns within `original` tokens, kept where it makes `high` or more, linear in the turns between
      ramp    factor, original, slow, fast        the same for `slow` and `fast` turns, linear in the pair's number between (from the last whole one before to the first behind), and all that is rotated times
              [amplitude]                         amplitude, 0.1 ln(factor) + 1 unless given
    The frequencies (`turns` of a full circle a position, float64) are made here once; a tensor of them may be given instead: turns, with amplitude."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, interleaved=False, scaling=None, turns=None, amplitude=1.0, device="cuda:0"):
        where = "Rotary"
        self.head_dim, self.rotary_dim, self.interleaved = head_dim, head_dim if rotary_dim is None else rotary_dim, bool(interleaved)
        n = self.rotary_dim
        if not (isinstance(head_dim, int) and 16 <= head_dim <= 1024 and head_dim % 16 == 0):
            _refuse(where, f"head_dim must be a multiple of 16 from 16 to 1024, got {head_dim}")
        if not (isinstance(n, int) and 16 <= n <= head_dim and n % 16 == 0):
            _refuse(where, f"rotary_dim must be a multiple of 16 from 16 to head_dim {head_dim}, got {n}")
        if turns is None:
            turns, much = _turns(n, base, scaling)
            self.turns, amplitude = torch.tensor(turns, dtype=torch.float64, device=device), amplitude * much
        else:
            if scaling is not None or not (isinstance(turns, torch.Tensor) and turns.is_cuda and turns.dtype == torch.float64 and turns.shape == (n // 2,) and turns.is_contiguous()):
                _refuse(where, f"turns must be a contiguous float64 tensor [{n // 2}] on the GPU, without a scaling")
            if turns.requires_grad:
                _refuse(where, "turns require a gradient, and a rotation has none")
            _no_gradient(where, "turns", turns)
            self.turns = turns
        if not self.turns.is_cuda:
            _refuse(where, "the device must be a GPU")
        if not math.isfinite(amplitude):
            _refuse(where, "the amplitude is not finite")
        self.amplitude, self.device = float(amplitude), self.turns.device
        self._index = self.device.index
        self._arg = pv_rotary(self.turns.data_ptr(), n, self.interleaved, self.amplitude)

    def rotate(self, x, positions, out=None, stream=None):
        """x [rows, heads, head_dim] (float32, bfloat16 or float16) turned by positions (int32 [rows]); out: where to (x itself, or memory that does not overlap it; made here otherwise)."""
        where = "Rotary.rotate"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.rotate(x, positions, out)
        xp, xr, xh = _heads(self, x, where, "x", None, _DTYPES)
        n, heads, hd = x.shape
        _positions(where, positions, n, self.device)
        if out is None:
            out = x.new_empty((n, heads, hd))
            op, orow, oh = out.data_ptr(), heads * hd, hd
        else:
            op, orow, oh = _heads(self, out, where, "out", heads, (x.dtype,))
            if out.shape[0] != n:
                _refuse(where, f"out must have {n} rows")
        rc = lib().pv_rotate(self._arg, positions.data_ptr(), xp, xr, xh, op, orow, oh, n, heads, hd, _DTYPES[x.dtype], _raw_stream(self._index))
        if rc:
            _check(rc, "pv_rotate")
        return out


_SCALINGS = {"linear": ("factor",), "base": ("factor",), "turns": ("factor", "original", "low", "high"), "ramp": ("factor", "original", "slow", "fast")}


def _turns(n, base, scaling):
    """Turns a position of each of n / 2 pairs, and the amplitude."""
    where = "Rotary"
    if not (base > 1 and math.isfinite(base)):
        _refuse(where, f"base must be a number above 1, got {base}")
    kind, much = None, 1.0
    if scaling is not None:
        kind = scaling.get("kind")
        if kind not in _SCALINGS or set(scaling) - {"kind", "amplitude"} != set(_SCALINGS[kind]) or ("amplitude" in scaling and kind != "ramp"):
            _refuse(where, f"scaling must be a kind with its numbers, one of {_SCALINGS}, got {scaling}")
        if not all(math.isfinite(scaling[k]) and scaling[k] > 0 for k in _SCALINGS[kind]):
            _refuse(where, f"the numbers of a scaling must be above 0, got {scaling}")
        s = scaling["factor"]
        if kind == "base":
            base = base * s ** (n / (n - 2))
    freq = [base ** (-2.0 * i / n) for i in range(n // 2)]
    if kind == "linear":
        freq = [f / s for f in freq]
    elif kind == "turns":
        low, high = scaling["low"], scaling["high"]
        if not low < high:
            _refuse(where, "low must be less than high")
        keep = [min(1.0, max(0.0, (scaling["original"] * f / (2 * math.pi) - low) / (high - low))) for f in freq]
        freq = [k * f + (1 - k) * f / s for k, f in zip(keep, freq)]
    elif kind == "ramp":
        if not scaling["slow"] < scaling["fast"]:
            _refuse(where, "slow must be less than fast")
        place = [n * math.log(scaling["original"] / (2 * math.pi * scaling[k])) / (2 * math.log(base)) for k in ("fast", "slow")]
        first, last = max(math.floor(place[0]), 0), min(math.ceil(place[1]), n - 1)
        keep = [1 - min(1.0, max(0.0, (i - first) / max(last - first, 0.001))) for i in range(n // 2)]
        freq = [k * f + (1 - k) * f / s for k, f in zip(keep, freq)]
        much = scaling.get("amplitude", 0.1 * math.log(s) + 1)
    return [f / (2 * math.pi) for f in freq], much


def _heads(self, t, where, name, heads, dtypes):
    """Rows [n, heads, head_dim], features next to each other: address and strides."""
    if not isinstance(t, torch.Tensor) or t.device != self.device:
        _refuse(where, f"{name} is not a tensor on {self.device}")
    shape, stride = t.shape, t.stride()
    if t.dtype not in dtypes or len(shape) != 3 or (heads is not None and shape[1] != heads) or shape[2] != self.head_dim:
        _refuse(where, f"{name} must be [rows, {'heads' if heads is None else heads}, {self.head_dim}] of {tuple(dtypes)}, got {tuple(shape)} of {t.dtype}")
    if stride[2] != 1:
        _refuse(where, f"{name}: the features of a head must lie next to each other")
    if _asks(t):
        _no_gradient(where, name, t)
    return t.data_ptr(), stride[0], stride[1]


def _positions(where, t, n, device):
    if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == torch.int32 and t.shape == (n,) and t.is_contiguous()):
        _refuse(where, f"positions must be a contiguous int32 tensor [{n}] on {device}")
    return t.data_ptr()


class KV16Pool:
    """Pages of a key/value cache in bfloat16 or float16 (dtype).  pages: the array ([n_pages, n_kv_heads, 2, page_tokens * head_dim] of dtype); made here unless given."""

    def __init__(self, n_pages, n_kv_heads, head_dim, page_tokens=16, dtype=torch.bfloat16, pages=None, device="cuda:0"):
        where = "KV16Pool"
        self.L = lib()
        if dtype not in _HALF:
            _refuse(where, f"dtype must be one of {tuple(_HALF)}")
        b = ctypes.c_size_t()
        _check(self.L.pv_kv16_bytes(ctypes.byref(pv_kv16_pool(None, n_pages, n_kv_heads, head_dim, page_tokens, _HALF[dtype])), ctypes.byref(b)), "pv_kv16_bytes")
        self.n_pages, self.n_kv_heads, self.head_dim, self.page_tokens, self.dtype = n_pages, n_kv_heads, head_dim, page_tokens, dtype
        shape = (n_pages, n_kv_heads, 2, page_tokens * head_dim)
        self.pages = torch.empty(shape, dtype=dtype, device=device) if pages is None else pages
        if not (isinstance(self.pages, torch.Tensor) and self.pages.is_cuda and self.pages.dtype == dtype and tuple(self.pages.shape) == shape and self.pages.is_contiguous()):
            _refuse(where, f"pages must be a contiguous {dtype} tensor {shape} on the GPU")
        if self.pages.requires_grad:
            _refuse(where, "pages require a gradient, and a cache has none")
        _no_gradient(where, "pages", self.pages)
        self.device = self.pages.device
        self._index = self.device.index
        self._arg = pv_kv16_pool(self.pages.data_ptr(), n_pages, n_kv_heads, head_dim, page_tokens, _HALF[dtype])
        self._need = {}                                    # (sequences, rows, heads, table's pages) -> bytes of attention's workspace

    def _seqs(self, seqs, where, n_rows):
        if not isinstance(seqs, KV8Seqs) or seqs.device != self.device:
            _refuse(where, f"seqs must be a KVSeqs on {self.device}")
        return seqs._arg(n_rows)

    def append(self, seqs, k, v, rotary=None, positions=None, q=None, q_out=None, stream=None):
        """Write k, v [rows, n_kv_heads, head_dim] (float32, bfloat16 or float16) into the pages of their sequences.  rotary: a Rotary that turns the keys on the way, by positions (int32 [rows]) or the tokens' own.  q [rows, heads,
        head_dim]: queries of the same rows and of k's type, turned alike and returned as such (q_out: where to, q itself if wanted; rows of no sequence are left as they are); attention() takes the pool's type, so
        that queries of another one have to be converted first."""
        where = "KV16Pool.append"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.append(seqs, k, v, rotary, positions, q, q_out)
        kp, kr, kh = _heads(self, k, where, "k", self.n_kv_heads, _DTYPES)
        vp, vr, vh = _heads(self, v, where, "v", self.n_kv_heads, _DTYPES)
        n = k.shape[0]
        if v.shape[0] != n or v.dtype != k.dtype:
            _refuse(where, "k and v must have the same rows and type")
        rot = None
        if rotary is not None:
            if not isinstance(rotary, Rotary) or rotary.device != self.device or rotary.head_dim != self.head_dim:
                _refuse(where, f"rotary must be a Rotary of heads of {self.head_dim} on {self.device}")
            rot = rotary._arg
        elif q is not None or positions is not None:
            _refuse(where, "queries and positions go with a rotary")
        at = None if positions is None else _positions(where, positions, n, self.device)
        qp, qr, qh, op, orow, oh, heads = 0, 0, 0, 0, 0, 0, 0
        if q is not None:
            qp, qr, qh = _heads(self, q, where, "q", None, (k.dtype,))
            heads = q.shape[1]
            if q.shape[0] != n:
                _refuse(where, f"q must have {n} rows")
            if q_out is None:
                q_out = q.new_empty((n, heads, self.head_dim))
                op, orow, oh = q_out.data_ptr(), heads * self.head_dim, self.head_dim
            else:
                op, orow, oh = _heads(self, q_out, where, "q_out", heads, (k.dtype,))
                if q_out.shape[0] != n:
                    _refuse(where, f"q_out must have {n} rows")
        elif q_out is not None:
            _refuse(where, "q_out goes with q")
        rc = self.L.pv_kv16_append(self._arg, self._seqs(seqs, where, n), kp, kr, kh, vp, vr, vh, rot, at, qp or None, qr, qh, heads, op or None, orow, oh, _DTYPES[k.dtype], _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv16_append")
        return q_out

    def attention(self, seqs, q, scale=None, mask=None, out=None, return_lse=False, lse=None, stream=None):
        """softmax(scale q K^T) V of every row of q [rows, n_q_heads, head_dim] (the pool's type) over its sequence's tokens; scale: 1 / sqrt(head_dim) unless given.  Without a mask a row sees the tokens up to its own
        position.  mask: int64 or uint64 [rows] or [rows, words], bit t % 64 of word t / 64: the row sees token prefix_len + t (a draft tree: its ancestors and itself), t less than the sequence's rows in the call; all tokens before
        prefix_len are seen.  Returns out, or (out, lse) with lse float32 [rows, n_q_heads]."""
        where = "KV16Pool.attention"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.attention(seqs, q, scale, mask, out, return_lse, lse)
        qp, qr, qh = _heads(self, q, where, "q", None, (self.dtype,))
        n, heads, _ = q.shape
        sa, mp, words = self._seqs(seqs, where, n), None, 0
        if mask is not None:
            if not (isinstance(mask, torch.Tensor) and mask.device == self.device and mask.dtype in (torch.int64, torch.uint64) and mask.dim() in (1, 2) and mask.shape[0] == n and mask.is_contiguous()):
                _refuse(where, f"mask must be a contiguous int64 tensor [{n}] or [{n}, words] on {self.device}")
            words = 1 if mask.dim() == 1 else mask.shape[1]
            if words == 0:
                _refuse(where, "mask must have a word a row")
            mp = mask.data_ptr()
        key = (sa.n_seq, n, heads, sa.table_pages)
        need = self._need.get(key)
        if need is None:
            b = ctypes.c_size_t()
            _check(self.L.pv_kv16_attention_bytes(self._arg, sa, heads, ctypes.byref(b)), "pv_kv16_attention_bytes")
            if len(self._need) > 256:
                self._need.clear()
            need = self._need[key] = b.value
        if out is None:
            out = q.new_empty((n, heads, self.head_dim))
            op, orow, oh = out.data_ptr(), heads * self.head_dim, self.head_dim
        else:
            op, orow, oh = _heads(self, out, where, "out", heads, (self.dtype,))
            if out.shape[0] != n:
                _refuse(where, f"out must have {n} rows")
        if lse is not None:
            if not (isinstance(lse, torch.Tensor) and lse.device == self.device and lse.dtype == torch.float32 and lse.shape == (n, heads) and lse.is_contiguous()):
                _refuse(where, f"lse must be a contiguous float32 tensor [{n}, {heads}] on {self.device}")
            if _asks(lse):
                _no_gradient(where, "lse", lse)
        elif return_lse:
            lse = q.new_empty((n, heads), dtype=torch.float32)
        ws = q.new_empty(need, dtype=torch.uint8) if need else None
        rc = self.L.pv_kv16_attention(self._arg, sa, qp, qr, qh, heads, mp, words, self.head_dim ** -0.5 if scale is None else scale, op, orow, oh, None if lse is None else lse.data_ptr(),
                                      None if ws is None else ws.data_ptr(), need, _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv16_attention")
        return out if lse is None else (out, lse)

    def keep(self, seqs, path, accepted, stream=None):
        """After a draft tree: the path's tokens (verify_drafts: path int32 [rows], accepted int32 [n_seq]) moved to where the sequence's rows began.  The prefix is accepted + 1 tokens longer then."""
        where = "KV16Pool.keep"
        if _elsewhere(self._index, stream):
            with _Elsewhere(self.device, stream):
                return self.keep(seqs, path, accepted)
        if not (isinstance(path, torch.Tensor) and path.device == self.device and path.dtype == torch.int32 and path.dim() == 1 and path.is_contiguous()):
            _refuse(where, f"path must be a contiguous int32 tensor [rows] on {self.device}")
        sa = self._seqs(seqs, where, path.shape[0])
        if not (isinstance(accepted, torch.Tensor) and accepted.device == self.device and accepted.dtype == torch.int32 and accepted.shape == (sa.n_seq,) and accepted.is_contiguous()):
            _refuse(where, f"accepted must be a contiguous int32 tensor [{sa.n_seq}] on {self.device}")
        rc = self.L.pv_kv16_keep(self._arg, sa, path.data_ptr(), accepted.data_ptr(), _raw_stream(self._index))
        if rc:
            _check(rc, "pv_kv16_keep")


_drafts_need = {}                                          # (rows, sequences, vocab) -> bytes of workspace


def verify_drafts(row_start, logits, tokens, u, draft_probs=None, parent=None, temperature=1.0, stream=None):
    """Which drafts the target takes, and the token that follows, by sampling: distributed as the target's own tokens are.  row_start (int32 [n + 1]): sequence s has rows row_start[s] .. row_start[s + 1] - 1; its first row's token
    is settled, each further one carries a draft.  logits [rows, vocab] (float32, bfloat16 or float16): the target's, of the token behind each row; tokens int32 [rows]; u float32 or float64 [rows, 2], random numbers from
    [0, 1): for taking the row's draft, for the draw behind the row.  A chain: the draft of row c is taken if u q < p of the row before it; draft_probs float32 [rows, vocab]: row c = the probabilities q that the
    draft of row c was drawn from (none: it was not drawn).  A tree: parent int32 [rows], the row of its sequence that the row hangs under (a lower number); a node's children are tried in order, none of them drawn.  temperature:
    a number, or float32 [n]; 0: the most probable token.  Returns accepted (int32 [n]: drafts taken), next_token (int32 [n]), path (int32 [rows]: the rows reached, from a sequence's first row on; None for a chain),
    probs (float32 [rows]: the target's probability of each draft)."""
    where = "verify_drafts"
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2 and logits.dtype in _DTYPES):
        _refuse(where, f"logits must be [rows, vocab] of {tuple(_DTYPES)} on the GPU")
    if _asks(logits):
        _no_gradient(where, "logits", logits)
    device = logits.device
    index = device.index
    if _elsewhere(index, stream):
        with _Elsewhere(device, stream):
            return verify_drafts(row_start, logits, tokens, u, draft_probs, parent, temperature)
    rows, vocab = logits.shape
    row_stride, one = logits.stride()
    if one != 1 and vocab > 1 and rows > 0:
        _refuse(where, "the logits of a row must lie next to each other")

    def ints(name, t, n):
        if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == torch.int32 and t.dim() == 1 and (n is None or t.shape[0] == n) and t.is_contiguous()):
            _refuse(where, f"{name} must be a contiguous int32 tensor [{'sequences + 1' if n is None else n}] on {device}")
        return t.data_ptr()
    start, tp = ints("row_start", row_start, None), ints("tokens", tokens, rows)
    n = row_start.shape[0] - 1
    if n < 0:
        _refuse(where, "row_start must have an entry")
    if not (isinstance(u, torch.Tensor) and u.device == device and u.dtype in (torch.float32, torch.float64) and u.shape == (rows, 2) and u.is_contiguous()):
        _refuse(where, f"u must be a contiguous float32 or float64 tensor [{rows}, 2] on {device}")
    qp, qr, pp = None, 0, None
    if parent is not None:
        if draft_probs is not None:
            _refuse(where, "a tree's drafts go without a drafter's probabilities")
        pp = ints("parent", parent, rows)
    if draft_probs is not None:
        if not (isinstance(draft_probs, torch.Tensor) and draft_probs.device == device and draft_probs.dtype == torch.float32 and draft_probs.shape == (rows, vocab)) or (draft_probs.stride(1) != 1 and vocab > 1 and rows > 0):
            _refuse(where, f"draft_probs must be a float32 tensor [{rows}, {vocab}] on {device}, a row's numbers next to each other")
        if _asks(draft_probs):
            _no_gradient(where, "draft_probs", draft_probs)
        qp, qr = draft_probs.data_ptr(), draft_probs.stride(0)
    hot, hp = 0.0, None
    if isinstance(temperature, torch.Tensor):
        if not (temperature.device == device and temperature.dtype == torch.float32 and temperature.shape == (n,) and temperature.is_contiguous()):
            _refuse(where, f"temperature must be a number or a contiguous float32 tensor [{n}] on {device}")
        if _asks(temperature):
            _no_gradient(where, "temperature", temperature)
        hp = temperature.data_ptr()
    else:
        hot = float(temperature)
    if _asks(u):
        _no_gradient(where, "u", u)
    L, key = lib(), (rows, n, vocab)
    need = _drafts_need.get(key)
    if need is None:
        b = ctypes.c_size_t()
        _check(L.pv_verify_drafts_bytes(rows, n, vocab, ctypes.byref(b)), "pv_verify_drafts_bytes")
        if len(_drafts_need) > 256:
            _drafts_need.clear()
        need = _drafts_need[key] = b.value
    # (one allocation for all that is returned)
    if parent is None:
        accepted, following, probs = logits.new_empty(2 * n + rows, dtype=torch.int32).split((n, n, rows))
        path = None
    else:
        accepted, following, probs, path = logits.new_empty(2 * n + 2 * rows, dtype=torch.int32).split((n, n, rows, rows))
    probs = probs.view(torch.float32)
    ws = logits.new_empty(need, dtype=torch.uint8) if need else None
    rc = L.pv_verify_drafts(start, n, logits.data_ptr(), row_stride, _DTYPES[logits.dtype], rows, vocab, tp, u.data_ptr(), u.dtype == torch.float64, qp, qr, pp, hp, hot,
                            accepted.data_ptr(), following.data_ptr(), None if path is None else path.data_ptr(), probs.data_ptr(), None if ws is None else ws.data_ptr(), need, _raw_stream(index))
    if rc:
        _check(rc, "pv_verify_drafts")
    return DraftVerdict(accepted, following, path, probs)
