"""Plain 64-bit model of the paged 8-bit KV cache and of filtered sampling (NumPy, one step per function).

Test infrastructure: it shares no code with the library.  `Cache` models the arrays of `jk_paged` and what
each call does to them, element by element; `tree_attention` is the attention over it; `sample_row` is the
sampling rule.
"""
from __future__ import annotations

import math

import numpy as np


# ------------------------------------------------------------------------------------------
# e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, 0x7f / 0xff are NaN
# ------------------------------------------------------------------------------------------
def e4m3_value(code: int) -> float:
    s, e, m = code >> 7, (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -v if s else v


E4M3 = np.array([e4m3_value(c) for c in range(256)])
_GRID = E4M3[:127]                                  # 0 .. 448, ascending with the code


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; past 448 the largest; NaN 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    hi = np.clip(np.searchsorted(_GRID, a), 0, 126)     # first grid value >= a (or the last)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _GRID[lo], _GRID[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    pick = np.where(a >= 448.0, 126, pick)
    code = pick.astype(np.uint8) | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), code).astype(np.uint8)


def block_scale(block: np.ndarray) -> float:
    """The smallest power of two s >= 2^-32 with max|x| <= 448 s over the finite values."""
    a = np.abs(np.asarray(block, dtype=np.float64))
    a = a[np.isfinite(a)]
    amax = float(a.max()) if a.size else 0.0
    s = 2.0 ** -32
    while amax > 448.0 * s:
        s *= 2.0
    return s


# ------------------------------------------------------------------------------------------
# the cache
# ------------------------------------------------------------------------------------------
class Refused(Exception):
    """The call changes nothing; args[0] is "BOUNDS" or "CAPACITY"."""


class Cache:
    def __init__(self, L, n_pages, ps, max_seqs, max_pages, Hkv, d):
        self.L, self.n_pages, self.ps, self.max_seqs, self.max_pages = L, n_pages, ps, max_seqs, max_pages
        self.Hkv, self.d = Hkv, d
        self.pages = np.zeros((2, L, n_pages, Hkv, ps, d), np.uint8)
        self.scale = np.zeros((2, L, n_pages, Hkv))
        self.open = np.zeros((2, L, max_seqs, Hkv, 2 * ps, d))
        self.kv_len = [0] * max_seqs
        self.table = [[-1] * max_pages for _ in range(max_seqs)]
        self.refcount = [0] * n_pages
        self.free = list(range(n_pages - 1, -1, -1))

    # requests: (row, first page, end) whose missing pages are to be taken, in order
    def _take(self, requests):
        missing = []
        for row, a, b in requests:
            for t in range(a, b):
                e = self.table[row][t]
                if e < 0:
                    missing.append((row, t))
                elif e >= self.n_pages or self.refcount[e] != 1:
                    raise Refused("BOUNDS")
        if len(missing) > len(self.free):
            raise Refused("CAPACITY")
        for row, t in missing:
            e = self.free.pop()
            self.table[row][t] = e
            self.refcount[e] = 1

    def _quantise(self, layers, kv, row, t, rows):
        """rows [len(layers), Hkv, ps, d] become page t of sequence `row`."""
        e = self.table[row][t]
        for j, layer in enumerate(layers):
            for h in range(self.Hkv):
                s = block_scale(rows[j, h])
                self.scale[kv, layer, e, h] = s
                self.pages[kv, layer, e, h] = e4m3_encode(rows[j, h] / s)

    def import_(self, seqs, n_tokens, first_layer, k_src, v_src):
        """k_src, v_src [layers, batch, Hkv, rows, d]"""
        rows = k_src.shape[3]
        if len(set(seqs)) < len(seqs):
            raise Refused("BOUNDS")
        for r, n in zip(seqs, n_tokens):
            if not 0 <= r < self.max_seqs or not 0 <= n <= min(rows, self.max_pages * self.ps):
                raise Refused("BOUNDS")
            if any(e >= 0 for e in self.table[r][n // self.ps:]):
                raise Refused("BOUNDS")
        self._take([(r, 0, n // self.ps) for r, n in zip(seqs, n_tokens)])
        layers = range(first_layer, first_layer + k_src.shape[0])
        for i, (r, n) in enumerate(zip(seqs, n_tokens)):
            for kv, src in ((0, k_src), (1, v_src)):
                for t in range(n // self.ps):
                    self._quantise(layers, kv, r, t, src[:, i, :, t * self.ps:(t + 1) * self.ps])
                for c in range(n // self.ps * self.ps, n):
                    self.open[kv, first_layer:first_layer + len(layers), r, :, c % (2 * self.ps)] = src[:, i, :, c]
            self.kv_len[r] = n

    def commit(self, k_tree, v_tree, n_acc, acc_idx, M):
        """k_tree, v_tree [L, B, Hkv, M, d]; kv_len counts the accepted nodes already."""
        requests = []
        for b, n in enumerate(n_acc):
            if n < 0:
                continue
            old = self.kv_len[b] - 1 - n
            if n >= M or old < 0 or self.kv_len[b] > self.max_pages * self.ps or any(
                    not 0 <= a < M for a in acc_idx[b][:n]):
                raise Refused("BOUNDS")
            requests.append((b, old // self.ps, self.kv_len[b] // self.ps))
        self._take(requests)
        for b, a, e in requests:
            nodes = [0] + list(acc_idx[b][:n_acc[b]])
            for kv, src in ((0, k_tree), (1, v_tree)):
                for j, node in enumerate(nodes):
                    c = self.kv_len[b] - 1 - n_acc[b] + j
                    self.open[kv, :, b, :, c % (2 * self.ps)] = src[:, b, :, node]
                for t in range(a, e):
                    half = (t % 2) * self.ps
                    self._quantise(range(self.L), kv, b, t, self.open[kv, :, b, :, half:half + self.ps])

    def fork(self, src, dst):
        ok = all(0 <= x < self.max_seqs for x in list(src) + list(dst))
        if not ok or len(set(dst)) < len(dst) or set(src) & set(dst):
            raise Refused("BOUNDS")
        if any(self.kv_len[x] or any(e >= 0 for e in self.table[x]) for x in dst):
            raise Refused("BOUNDS")
        for s, t in zip(src, dst):
            nf = self.kv_len[s] // self.ps
            self.table[t][:nf] = self.table[s][:nf]
            for e in self.table[s][:nf]:
                self.refcount[e] += 1
            self.kv_len[t] = self.kv_len[s]
            for c in range(nf * self.ps, self.kv_len[s]):
                self.open[:, :, t, :, c % (2 * self.ps)] = self.open[:, :, s, :, c % (2 * self.ps)]

    def release(self, seqs):
        if len(set(seqs)) < len(seqs) or any(not 0 <= r < self.max_seqs for r in seqs):
            raise Refused("BOUNDS")
        empty = set()
        for r in seqs:
            for e in self.table[r]:
                if e >= 0:
                    self.refcount[e] -= 1
                    if self.refcount[e] == 0:
                        empty.add(e)
            self.table[r] = [-1] * self.max_pages
            self.kv_len[r] = 0
        self.free += sorted(empty)

    def compact(self):
        live = sum(c > 0 for c in self.refcount)
        movers = [e for e in range(live, self.n_pages) if self.refcount[e] > 0]
        holes = [e for e in range(live) if self.refcount[e] == 0]
        for s, t in zip(movers, holes):
            self.pages[:, :, t] = self.pages[:, :, s]
            self.scale[:, :, t] = self.scale[:, :, s]
            self.refcount[t], self.refcount[s] = self.refcount[s], 0
            self.table = [[t if e == s else e for e in row] for row in self.table]
        self.free = list(range(self.n_pages - 1, live - 1, -1))
        return len(movers)

    def columns(self, kv, layer, b, h, tree):
        """The committed tokens of sequence b and the tree's rows, as numbers [kv_len + M, d]."""
        n, ps = self.kv_len[b], self.ps
        rows = []
        for c in range(n):
            if c < n // ps * ps:
                e = self.table[b][c // ps]
                rows.append(E4M3[self.pages[kv, layer, e, h, c % ps]] * self.scale[kv, layer, e, h])
            else:
                rows.append(self.open[kv, layer, b, h, c % (2 * ps)])
        return np.array(rows + list(tree), dtype=np.float64)


def tree_attention(cache: Cache, layer, q, k_tree, v_tree, parent, scale):
    """q [B, M, Hq, d], k_tree, v_tree [B, Hkv, M, d], parent [B, M].  Returns (out, size): size is
    sum_c p_c |v_c|, what a relative error of the weights is measured against."""
    B, M, Hq, d = q.shape
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    G = Hq // cache.Hkv
    for b in range(B):
        n = cache.kv_len[b]
        seen = np.zeros((M, n + M), bool)
        seen[:, :n] = True
        for i in range(M):
            j = i
            while j >= 0:
                seen[i, n + j] = True
                j = parent[b, j]
        for h in range(cache.Hkv):
            k = cache.columns(0, layer, b, h, k_tree[b, h])
            v = cache.columns(1, layer, b, h, v_tree[b, h])
            for g in range(h * G, (h + 1) * G):
                z = np.where(seen, (q[b, :, g].astype(np.float64) @ k.T) * scale, -np.inf)
                p = np.exp(z - z.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[b, :, g] = p @ v
                size[b, :, g] = p @ np.abs(v)
    return out, size


# ------------------------------------------------------------------------------------------
# sampling
# ------------------------------------------------------------------------------------------
def sample_row(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, kept mask) of one row; the per-row parameters are the fp32 values the device is given."""
    z = np.asarray(z, dtype=np.float64).copy()
    z[np.isnan(z)] = -np.inf
    z[z == np.inf] = np.float64(np.finfo(np.float32).max)
    kept = np.zeros(len(z), bool)
    if not np.any(z > -np.inf):
        return -1, kept
    order = np.lexsort((np.arange(len(z)), -z))                  # logit descending, index ascending
    order = [i for i in order if z[i] > -np.inf]
    if not temperature > 0:
        kept[order[0]] = True
        return int(order[0]), kept
    zmax = z[order[0]]
    w = np.exp((z[order] - zmax) / temperature)
    n = len(order)
    k = min(top_k, n) if top_k > 0 else n
    keep = k
    if top_p < 1:
        target = top_p * math.fsum(w[:k])
        before = np.concatenate([[0.0], np.cumsum(w[:k])[:-1]])
        keep = min(keep, int(np.sum(before < target)))
    if min_p > 0:
        keep = min(keep, int(np.sum(z[order] - zmax >= temperature * math.log(min_p))))
    order = order[:max(1, keep)]
    kept[order] = True
    idx = np.flatnonzero(kept)
    c = np.cumsum(np.exp((z[idx] - zmax) / temperature))
    hit = np.flatnonzero(c > u * c[-1])
    return int(idx[hit[0]] if len(hit) else idx[-1]), kept
