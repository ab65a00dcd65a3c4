"""One row of the decoder over 8-bit K/V in 64 bits (tests only): the cached-context decoder of the
reference with every layer's keys and values held by the 8-bit cache's reference."""
import math

import numpy as np

import oracle.decoder as D
import oracle.qcache as Q


class QuantRow:
    """Steps with given fed-back bins; `select`: pages that a decode query attends to (0: all).

    margin: the smallest relative gap met between the last chosen page's score and the first one left out;
    units: the same gap in whole numbers of the score (of the largest key scale among the row's pages).
    """

    def __init__(self, p, capacity, select=0):
        self.p, self.select, self.margin, self.units = p, select, math.inf, math.inf
        c = p.cfg
        n = capacity // 64
        z = lambda *s: np.zeros((n, c.n_heads) + s, np.uint8)  # noqa: E731
        self.layers = [Q.Cache(z(64, c.head_dim), z(16, c.head_dim, 4), np.zeros((n, c.n_heads), np.int64),
                               np.zeros((n, c.n_heads), np.int64), np.zeros((n, c.n_heads, 2, c.head_dim), np.int64),
                               np.arange(n, dtype=np.int32)[None]) for _ in range(c.n_layers)]
        self.len, self.h_last = 0, None

    def forward(self, x, start, decode=False):
        c, p = self.p.cfg, self.p
        h = np.asarray(x, dtype=np.float64)
        pos = np.arange(start, start + len(h))
        for l, cache in enumerate(self.layers):
            u = D.rms_norm(h, p.layer("g_attn", l), c.rms_eps)
            q, k, v = (D.split_heads(D.linear(p.layer(n, l), u), c) for n in ("w_q", "w_k", "w_v"))
            q, k = D.apply_rope(q, pos, c.rope_theta), D.apply_rope(k, pos, c.rope_theta)
            Q.append(cache, 0, start, k, v)
            o = np.zeros_like(q)
            for t in range(len(h)):
                for a in range(c.n_heads):
                    pages = None
                    if decode and self.select:
                        pages = Q.select(cache, 0, a, q[t, a][None], int(pos[t]) + 1, self.select)
                        self._gap(cache, a, q[t, a], int(pos[t]) + 1, pages)
                    o[t, a] = Q.attend(cache, 0, a, q[t, a][None], int(pos[t]) + 1, 1 / math.sqrt(c.head_dim), pages)[0][0]
            h = h + D.linear(p.layer("w_o", l), o.reshape(len(h), c.d_model))
            u = D.rms_norm(h, p.layer("g_ffn", l), c.rms_eps)
            h = h + D.linear(p.layer("w_down", l), D.silu(D.linear(p.layer("w_gate", l), u)) * D.linear(p.layer("w_up", l), u))
        return h

    def _gap(self, cache, head, q, vis, pages):
        n = -(-vis // 64)
        if n <= self.select:
            return
        top = math.frexp(float(np.abs(q).max()))[1]
        w = np.clip(np.rint(q * 2.0 ** (7 - top)), -127, 127)
        s = [float(np.maximum(w, 0) @ cache.bounds[i, head, 0] + np.minimum(w, 0) @ cache.bounds[i, head, 1]) * 2.0 ** cache.ke[i, head]
             for i in range(n - 1)]
        kept, left = [s[i] for i in pages if i < n - 1], [s[i] for i in range(n - 1) if i not in pages]
        if kept and left:
            self.margin = min(self.margin, (min(kept) - max(left)) / max(map(abs, s)))
            self.units = min(self.units, (min(kept) - max(left)) * 2.0 ** -int(cache.ke[:n, head].max()))

    def commit(self, x):
        if x is not None and len(x):
            h = self.forward(x, self.len)
            self.len += len(x)
            self.h_last = h[-1]

    def step(self, new, fed):
        self.commit(new)
        z, h = [], self.h_last
        for j in range(len(fed)):
            z.append(D.bin_logits(self.p, h))
            if j + 1 < len(fed):
                h = self.forward(D.bin_embedding(self.p, int(fed[j]))[None], self.len + j, decode=True)[-1]
        return np.stack(z)
