"""A decoder in 64 bits over an 8-bit key/value cache: the public LLaMA definition in numpy, keys and values rounded to bf16 and then stored by tests/kv8_ref.py's rule."""
import numpy as np

import kv8_ref
import pv_inputs
from helpers import tensors_f64


def bf16(x):
    return pv_inputs.bf16_bits_to_f32(pv_inputs.bf16_round_f32(x.astype(np.float32))).astype(np.float64)


class Decoder:
    def __init__(self, shape, gains="ones", max_tokens=512, tensors=None):
        self.s, self.t = shape, tensors or tensors_f64(shape, gains)
        pages = -(-max_tokens // shape.page_tokens)
        self.table = np.arange(pages)
        z = lambda *d: np.zeros(d, np.uint8)  # noqa: E731
        self.pools = [kv8_ref.Pool(z(pages, shape.n_kv_heads, 2, shape.page_tokens * shape.head_dim), z(pages, shape.n_kv_heads, shape.page_tokens // 16, 2), shape.head_dim, shape.page_tokens)
                      for _ in range(shape.n_layers)]
        self.len, self.pending = 0, -1

    def norm(self, x, g):
        return x / np.sqrt((x * x).mean(1, keepdims=True) + self.s.rms_eps) * g.reshape(1, -1)

    def rotated(self, x, pos):
        half = self.s.head_dim // 2
        a = pos[:, None] * self.s.rope_base ** (-2.0 * np.arange(half) / self.s.head_dim)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        u, v = x[..., :half], x[..., half:]
        return np.concatenate([u * c - v * s, v * c + u * s], -1)

    def forward(self, tokens, parents=None):
        """Logits of a block behind the committed tokens (which stay as many); parents: a draft tree."""
        s, n, T = self.s, len(tokens), self.len
        par = np.arange(-1, n - 1) if parents is None else np.asarray(parents)
        see, depth = np.zeros((n, n), bool), np.zeros(n, int)
        for i in range(n):
            if par[i] >= 0:
                see[i], depth[i] = see[par[i]], depth[par[i]] + 1
            see[i, i] = True
        see = np.concatenate([np.ones((n, T), bool), see], 1)
        pos = T + depth
        x = self.t["embed", -1].reshape(s.vocab, s.d_model)[np.asarray(tokens)]
        group = s.n_q_heads // s.n_kv_heads
        for l in range(s.n_layers):
            w = lambda k: self.t[k, l]  # noqa: E731
            a = self.norm(x, w("attn_norm"))
            q, k, v = ((a @ w(m).T).reshape(n, -1, s.head_dim) for m in ("wq", "wk", "wv"))
            q, k = self.rotated(q, pos), self.rotated(k, pos)
            self.pools[l].append([0, n], [T], [self.table], bf16(k), bf16(v))
            ks, vs, _ = self.pools[l].tokens(self.table, 0, T + n)
            out = np.empty_like(q)
            for h in range(s.n_q_heads):
                sc = np.where(see, q[:, h] @ ks[:, h // group].T / np.sqrt(s.head_dim), -np.inf)
                p = np.exp(sc - sc.max(1, keepdims=True))
                out[:, h] = p / p.sum(1, keepdims=True) @ vs[:, h // group]
            x = x + out.reshape(n, -1) @ w("wo").T
            a = self.norm(x, w("ffn_norm"))
            g = a @ w("wg").T
            x = x + (g / (1 + np.exp(-g)) * (a @ w("wu").T)) @ w("wd").T
        return self.norm(x, self.t["final_norm", -1]) @ self.t["lm_head", -1].reshape(s.vocab, s.d_model).T

    def prefill(self, tokens, chunk=64):
        for i in range(0, len(tokens), chunk):
            lg = self.forward(tokens[i:i + chunk])
            self.len += len(tokens[i:i + chunk])
        self.pending = int(lg[-1].argmax())
        return lg[-1]

    def verify(self, draft):
        lg = self.forward(draft)
        pred = lg.argmax(1)
        n = 0
        while n < len(draft) and draft[n] == (pred[n - 1] if n else self.pending if self.pending >= 0 else draft[0]):
            n += 1
        self.len += n
        self.pending = int(pred[n - 1]) if n else self.pending
        return n, self.pending, pred, lg

    def rollback(self, n):
        self.len, self.pending = n, -1

    def export(self):
        kv = [p.tokens(self.table, 0, self.len)[:2] for p in self.pools]
        return np.array(kv).reshape(self.s.n_layers, 2, self.len, -1)
