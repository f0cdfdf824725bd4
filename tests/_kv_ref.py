"""Plain 64-bit forms of the paged 8-bit cache's operators, and caches to run them on."""
import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn


def frequencies(rotary, base=10000.0, scaling="none", factor=1.0, context=0):
    """(radians a position [rotary/2], magnitude) as include/esp_kv.h defines them."""
    out = []
    if scaling == "ntk":
        base = base * factor ** (rotary / (rotary - 2))
    for i in range(rotary // 2):
        f = base ** (-2 * i / rotary)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            share = min(1.0, max(0.0, (f * context / (2 * math.pi) - 1) / 31))
            f *= share + (1 - share) / factor
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0)


def rotate(x, positions, f, magnitude, interleaved, inverse=False):
    """x [tokens, heads, dim] float64 (numpy)."""
    x, y = np.asarray(x, np.float64), np.array(x, np.float64)
    n = len(f)
    angle = np.asarray(positions, np.float64)[:, None, None] * f * (-1 if inverse else 1)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y[..., a] = magnitude * (x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle))
    y[..., b] = magnitude * (x[..., a] * np.sin(angle) + x[..., b] * np.cos(angle))
    return y


def host(cache, layer=0):
    """Numbers of a cache's pages: k [P][H][T][D], v [P][H][T][D] float64, from its codes and scales."""
    s = cache.scale[:, layer].double().cpu().numpy()
    k = cache.k.view(torch.uint8)[:, layer].contiguous().cpu().view(F8).double().numpy() * s[:, 0, :, None, None]
    v = cache.v.view(torch.uint8)[:, layer].contiguous().cpu().view(F8).double().numpy().swapaxes(-1, -2) * s[:, 1, :, None, None]
    return k, v


def tokens_of(pool, table, length):
    """[length][H][D] of one sequence."""
    T = pool.shape[2]
    x = pool[table[:-(-length // T)]].swapaxes(1, 2)
    return x.reshape(-1, *x.shape[2:])[:length]


def attend(q, k, v, n, window, scale):
    """q [n][Hq][D], k, v [L][H][D] float64 -> out, lse, spread: sum p |v|, most: max sum |q k| scale."""
    L, H = k.shape[0], k.shape[1]
    G = q.shape[1] // H
    out, lse = np.zeros_like(q), np.full(q.shape[:2], -np.inf)
    spread, most = np.zeros_like(q), 0.0
    for i in range(n):
        p = L - n + i
        lo, hi = (max(0, p - window + 1) if window else 0), p + 1
        if hi <= lo:
            continue
        for h in range(q.shape[1]):
            kk, vv = k[lo:hi, h // G], v[lo:hi, h // G]
            s = scale * (kk @ q[i, h])
            most = max(most, float(np.nanmax(np.abs(kk) @ np.abs(q[i, h])) * abs(scale)))
            m = s.max()
            w = np.exp(s - m)
            out[i, h] = (w @ vv) / w.sum()
            spread[i, h] = (w @ np.abs(vv)) / w.sum()
            lse[i, h] = m + np.log(w.sum())
    return out, lse, spread, most


def make(kv, lengths, pages=None, page=16, heads=2, dim=64, layers=1, width=None, seed=0, spare=3):
    """A cache of sequences of these lengths on pages from all over the pool.  Every code and scale that belongs to no
    token is NaN."""
    g = np.random.default_rng(seed)
    counts = [-(-n // page) for n in lengths]
    P = pages or sum(counts) + spare
    W = width or max(1, max(counts))
    order = g.permutation(P)
    k = (g.standard_normal((P, layers, heads, page, dim)) * 90).clip(-448, 448).astype(np.float32)
    v = (g.standard_normal((P, layers, heads, dim, page)) * 90).clip(-448, 448).astype(np.float32)
    scale = np.exp2(g.integers(-9, -5, (P, layers, 2, heads))).astype(np.float32)
    table, refs, at = np.full((len(lengths), W), -1, np.int32), np.zeros(P, np.int32), 0
    used = np.zeros((P, page), bool)
    for s, (n, c) in enumerate(zip(lengths, counts)):
        table[s, :c] = order[at:at + c]
        refs[order[at:at + c]] += 1
        for j in range(c):
            used[table[s, j], :min(page, n - j * page)] = True
        at += c
    kc, vc = (torch.from_numpy(x).to(F8).view(torch.uint8).numpy() for x in (k, v))
    kc[np.broadcast_to(~used[:, None, None, :, None], kc.shape)] = 0x7f
    vc[np.broadcast_to(~used[:, None, None, None, :], vc.shape)] = 0xff
    scale[~used.any(1)] = np.nan
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    return kv.PagedCache.adopt(dev(kc).view(F8), dev(vc).view(F8), dev(scale), dev(table),
                               torch.tensor(lengths, dtype=torch.int32, device="cuda"), dev(refs))


def offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")


class Pages:
    """The page operations on host integers; `names` follows every page's contents."""

    def __init__(self, cache):
        self.table, self.lengths, self.refs = (t.cpu().numpy().copy() for t in (cache.table, cache.lengths, cache.refs))
        self.T, self.names = cache.page_tokens, np.arange(len(self.refs))

    def _free(self, n):
        return np.nonzero(self.refs == 0)[0][:n]

    def resize(self, lengths):
        T = self.T
        old = self.table.copy(), self.refs.copy()
        for s, n in enumerate(lengths):
            for j in range(-(-n // T), self.table.shape[1]):
                if self.table[s, j] >= 0:
                    self.refs[self.table[s, j]] -= 1
                    self.table[s, j] = -1
        need = []
        for s, n in enumerate(lengths):
            for j in range(-(-n // T)):
                p, last = self.table[s, j], min(n, self.lengths[s])
                if p < 0 or (j == last // T and last % T and self.refs[p] > 1):
                    need.append((s, j, p))
        free = self._free(len(need))
        if len(free) < len(need):
            self.table, self.refs = old
            return False
        for (s, j, p), f in zip(need, free):
            if p >= 0:
                self.names[f] = self.names[p]
        for (s, j, p), f in zip(need, free):
            if p >= 0:
                self.refs[p] -= 1
            self.refs[f] = 1
            self.table[s, j] = f
        self.lengths = np.array(lengths, np.int32)
        return True

    def fork(self, parents, children):
        T = self.T
        old = self.table.copy(), self.refs.copy()
        for c in children:
            for p in self.table[c][self.table[c] >= 0]:
                self.refs[p] -= 1
        part = [self.lengths[p] % T > 0 for p in parents]
        free = self._free(sum(part))
        if len(free) < sum(part):
            self.table, self.refs = old
            return False
        at = 0
        for p, c, copy in zip(parents, children, part):
            row = self.table[p].copy()
            j = self.lengths[p] // T
            if copy:
                self.names[free[at]] = self.names[row[j]]
                row[j] = free[at]
                at += 1
            for page in row[row >= 0]:
                self.refs[page] += 1
            self.table[c], self.lengths[c] = row, self.lengths[p]
        return True

    def compact(self, limit=None):
        live = np.nonzero(self.refs > 0)[0]
        limit = len(live) if limit is None else min(limit, len(self.refs))
        if len(live) > limit:
            return False
        source, to = live[live >= limit], [p for p in range(limit) if self.refs[p] == 0]
        for a, b in zip(source, to):
            self.names[b] = self.names[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b
        return True
