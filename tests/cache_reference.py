"""Plain float64 reference of the 8-bit paged cache (include/tppsd.h): page
bookkeeping, the 8-bit form of whole blocks and causal attention, sequence by
sequence."""
import numpy as np
import torch

BLOCK, RING, E_MIN = 64, 128, -100
CAPACITY, PAGES, SEQUENCE, OPEN = 1, 8, 16, 32


def e4m3(x):
    """Block x [BLOCK, KV, dh] (float64) as its codes and scale stand for it, per head."""
    fin = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=(0, 2), keepdims=True)
    m, e = np.frexp(fin)                                  # fin = m 2^e; fin <= 448 2^(e - 9) iff m <= 0.875
    e = np.where(fin > 0, np.maximum(np.where(m <= 0.875, e - 9, e - 8), E_MIN), 0)
    y = np.ldexp(np.where(np.isfinite(x), x, 0.0), -e)
    step = np.ldexp(1.0, np.maximum(np.frexp(y)[1] - 1, -6) - 3)
    return np.where(np.isfinite(x), np.ldexp(np.round(y / step) * step, e), np.nan)


class CacheRef:
    def __init__(self, L, H, KV, dh, S, max_events, n_pages=0):
        self.L, self.H, self.KV, self.dh, self.S, self.max_events = L, H, KV, dh, S, max_events
        self.NP = -(-max_events // BLOCK)
        self.n_pages = n_pages or self.NP * S
        self.table = np.full((S, self.NP), -1)
        self.refs = np.zeros(self.n_pages, dtype=int)
        self.lens, self.held, self.low, self.pend = (np.zeros(S, dtype=int) for _ in range(4))
        self.rows = np.zeros((S, 2, L, max_events, KV, dh))      # rows as they came
        self.status = 0

    def _free(self):
        return [int(p) for p in np.nonzero(self.refs == 0)[0]]

    def _drop(self, s, j0):
        for j in range(j0, self.held[s]):
            self.refs[self.table[s, j]] -= 1
            self.table[s, j] = -1
        self.held[s] = min(self.held[s], j0)

    def begin(self, B, n_new, seqs=None, counts=None):
        seqs = range(B) if seqs is None else seqs
        free, off = self._free(), 0
        self.plan, self.P, named = [], n_new, set()
        for i, s in enumerate(seqs):
            if not 0 <= s < self.S or s in named:
                self.status |= SEQUENCE
                self.plan.append((-1, 0, 0))
                continue
            named.add(s)
            start, cnt = int(self.lens[s]), n_new if counts is None else min(max(int(counts[i]), 0), n_new)
            if cnt and start + cnt > self.max_events:
                self.status |= CAPACITY
                cnt = 0
            need = max(0, (start + cnt) // BLOCK - int(self.held[s])) if cnt else 0
            if need:
                if off + need <= len(free):
                    for p in free[off:off + need]:
                        self.table[s, self.held[s]] = p
                        self.refs[p] = 1
                        self.held[s] += 1
                else:
                    self.status |= PAGES
                    cnt = 0
                off += need
            self.pend[s] = cnt
            if cnt:
                if start % BLOCK and start // BLOCK < self.low[s]:
                    self.status |= OPEN
                top = (start + cnt - 1) // BLOCK
                self.low[s] = max(top - 1, min(self.low[s], start // BLOCK))
            self.plan.append((s, start, cnt))

    def append(self, layer, k, v):
        for i, (s, start, cnt) in enumerate(self.plan):
            if s >= 0 and cnt:
                self.rows[s, 0, layer, start:start + cnt] = k[i, :cnt]
                self.rows[s, 1, layer, start:start + cnt] = v[i, :cnt]

    def held_rows(self, s, side, layer, end):
        x = self.rows[s, side, layer, :end].copy()
        for a in range(0, end // BLOCK * BLOCK, BLOCK):
            x[a:a + BLOCK] = e4m3(x[a:a + BLOCK])
        return x

    def attend(self, layer, q, out, scale, sink):
        """Rows of `out` [B, P, H, dh] in place; returns, per element, what the
        output's error is measured by: the mean of |V| under the weights
        ("weight"), and the largest sum of |q k| scale of the row ("score")."""
        weight, score = np.zeros(out.shape), np.zeros(out.shape)
        G = self.H // self.KV
        for i, (s, start, cnt) in enumerate(self.plan):
            if s < 0 or not cnt:
                continue
            end = start + cnt
            came = [self.rows[s, side, layer, :end] for side in (0, 1)]
            held = [self.held_rows(s, side, layer, end) for side in (0, 1)]
            for p in range(cnt):
                a = (start + p) // BLOCK * BLOCK
                kk = np.concatenate([held[0][:a], came[0][a:start + p + 1]])
                vv = np.concatenate([held[1][:a], came[1][a:start + p + 1]])
                for h in range(self.H):
                    sc = kk[:, h // G] @ q[i, p, h] * scale
                    m = max(sc.max(), 0.0) if sink else sc.max()
                    w = np.exp(sc - m)
                    tot = w.sum() + (np.exp(-m) if sink else 0.0)
                    out[i, p, h] = w @ vv[:, h // G] / tot
                    weight[i, p, h] = w @ np.abs(vv[:, h // G]) / tot
                    score[i, p, h] = (np.abs(kk[:, h // G]) @ np.abs(q[i, p, h]) * scale).max()
        return weight, score

    def _settle(self, s, n):
        if n % BLOCK and n // BLOCK < self.low[s]:
            self.status |= OPEN
            n = n // BLOCK * BLOCK
        return n

    def commit(self, accept=None):
        for i, (s, start, cnt) in enumerate(self.plan):
            if s >= 0 and cnt:
                a = cnt if accept is None else min(max(int(accept[i]), 0), cnt)
                self.lens[s], self.pend[s] = self._settle(s, start + a), 0

    def truncate(self, seqs, lens=None):
        for i, s in enumerate(seqs):
            n = 0 if lens is None else int(lens[i])
            if not 0 <= s < self.S or n < 0:
                self.status |= SEQUENCE
                continue
            if n >= self.lens[s]:
                n = int(self.lens[s])
            else:
                n = self._settle(s, n)
            self.lens[s], self.pend[s] = n, 0
            self._drop(s, n // BLOCK)

    def _pairs(self, other, src, dst, same):
        good, named = [], set()
        for s, d in zip(src, dst):
            ok = 0 <= s < other.S and 0 <= d < self.S
            if ok and d in named:
                ok = False
            if 0 <= s < other.S and 0 <= d < self.S:
                named.add(d)
            if ok and same and any(d == x for x, y in zip(src, dst) if 0 <= x < other.S and 0 <= y < self.S):
                ok = False
            if not ok:
                self.status |= SEQUENCE
            elif other.lens[s] > self.max_events:
                self.status |= CAPACITY
                ok = False
            if ok:
                good.append((s, d))
        return good

    def _take(self, d, other, s):
        n = int(other.lens[s])
        if n % BLOCK and n // BLOCK < other.low[s]:
            self.status |= OPEN
        self.rows[d, :, :, :n] = other.rows[s, :, :, :n]
        self.lens[d], self.held[d], self.low[d], self.pend[d] = n, n // BLOCK, n // BLOCK, 0

    def fork(self, src, dst):
        good = self._pairs(self, src, dst, True)
        for s, d in good:
            self._drop(d, 0)
        for s, d in good:
            n = int(self.lens[s]) // BLOCK
            self.table[d, :n] = self.table[s, :n]
            self.refs[self.table[s, :n]] += 1
            self._take(d, self, s)

    def copy(self, other, src, dst):
        good = self._pairs(other, src, dst, False)
        for s, d in good:
            self._drop(d, 0)
            self.lens[d] = self.held[d] = self.low[d] = self.pend[d] = 0
        used = sorted({int(p) for s, d in good for p in other.table[s, :other.lens[s] // BLOCK]})
        free = self._free()
        if len(used) > len(free):
            self.status |= PAGES
            return
        to = dict(zip(used, free))
        for s, d in good:
            n = int(other.lens[s]) // BLOCK
            for j in range(n):
                self.table[d, j] = to[int(other.table[s, j])]
                self.refs[self.table[d, j]] += 1
            self._take(d, other, s)


def tolerance(prec, dh, keys, out, weight, score):
    """Bound of |kernel - float64| per element, from the roundings alone.

    Scores: products of dh terms summed in fp32, times the scale, less the
    maximum: (dh + 4) 2^-24 sum |q k| scale absolute, as much relative in the
    weight; both the weight and the normaliser carry it. exp2: 2^-22. bf16: each
    weight rounds by 2^-8 in numerator and normaliser alike, so the output moves
    by at most 2^-8 (mean |V| + |o|), and the output itself rounds by 2^-8. fp32:
    three bf16 parts hold a weight to 2^-24, sums over the keys in fp32 err by
    less than keys 2^-24 of the mean |V|."""
    u = 2.0 ** -24
    soft = 2 * ((dh + 4) * u * score + 2.0 ** -22)
    if prec == "bf16":
        return weight * (2.0 ** -8 + soft + keys * u) + np.abs(out) * (2 * 2.0 ** -8 + soft)
    return weight * (soft + (2 * keys + 16) * u) + np.abs(out) * (soft + (keys + 16) * u)


def values(t):
    """A tensor's values as a float64 array."""
    return t.detach().to(torch.float64).cpu().numpy()
