"""The float64 oracle model with the target's keys and values in the 8-bit
paged cache (TPPSD_FLAG_CACHE8): position i attends to the blocks of 64 before
its own as e4m3 with a power-of-two scale per block and head stand for them,
and to its own block as it came."""
import math

import numpy as np

from cache_reference import BLOCK, e4m3
from oracle.model import Model


class Model8(Model):
    """jitter: relative size of a random change of every key and value before
    they are cached, for how far roundings of that size carry to the outputs."""

    def __init__(self, cfg, weights, jitter=0.0, seed=0):
        super().__init__(cfg, weights)
        self.jitter, self.rng = jitter, np.random.default_rng(seed)

    def _mix(self, q, K, V, pos, sink):
        """q [B, H, P, dh] at positions pos [B, P] over rows K, V [B, H, N, dh]."""
        B, H, N, dh = K.shape
        whole = N // BLOCK * BLOCK
        held = []
        for x in (K, V):
            h = x.copy()
            for a in range(0, whole, BLOCK):
                h[:, :, a:a + BLOCK] = np.stack([np.moveaxis(e4m3(np.moveaxis(x[b, :, a:a + BLOCK], 0, 1)), 1, 0)
                                                 for b in range(B)])
            held.append(h)
        j, i = np.arange(N)[None, None], pos[:, :, None]
        before = (j // BLOCK < i // BLOCK)[:, None]
        own = ((j // BLOCK == i // BLOCK) & (j <= i))[:, None]
        s8, s = (q @ np.swapaxes(x, -1, -2) / math.sqrt(dh) for x in (held[0], K))
        sc = np.where(before, s8, np.where(own, s, -np.inf))
        m = sc.max(axis=-1, keepdims=True)
        if sink:
            m = np.maximum(m, 0.0)
        p = np.exp(sc - m)
        tot = p.sum(axis=-1, keepdims=True) + (np.exp(-m) if sink else 0.0)
        return (np.where(before, p, 0.0) @ held[1] + np.where(own, p, 0.0) @ V) / tot

    def forward_block(self, cache, t, k, pos0, rows=None):
        rb, d = self.rb, self.d
        t = np.asarray(t)
        B, P = t.shape
        pos = np.asarray(pos0, dtype=np.int64)[:, None] + np.arange(P)[None]
        rows = np.arange(B) if rows is None else np.asarray(rows, dtype=np.int64)
        N = int(pos.max()) + 1
        x, z = self.embed(t, k), self.time_encoding(t)
        for l in range(self.L):
            p = f"layers.{l}."
            if self.attnhp:
                a = np.concatenate([rb(z), rb(x)], axis=-1)
            else:
                a = rb(self.layer_norm(x, self.w[p + "ln1.g"], self.w[p + "ln1.b"]))
            qkv = rb(self._lin(a, p + "qkv"))
            q, kk, v = (self._split_heads(qkv[..., i * d:(i + 1) * d]) for i in range(3))
            for store, new in ((cache.K[l], kk), (cache.V[l], v)):
                if self.jitter:
                    new = rb(new * (1.0 + self.jitter * self.rng.uniform(-1, 1, new.shape)))
                store[rows[:, None], :, pos, :] = np.moveaxis(new, 1, 2)
            o = rb(self._merge_heads(self._mix(q, cache.K[l][rows, :, :N], cache.V[l][rows, :, :N], pos, self.attnhp)))
            if self.attnhp:
                x = x + np.tanh(o)
                continue
            x = x + self._lin(o, p + "out")
            a = rb(self.layer_norm(x, self.w[p + "ln2.g"], self.w[p + "ln2.b"]))
            x = x + self._lin(rb(np.maximum(self._lin(a, p + "ffn1"), 0.0)), p + "ffn2")
        return x if self.attnhp else self.layer_norm(x, self.w["lnf.g"], self.w["lnf.b"])
