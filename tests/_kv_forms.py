"""Plain 64-bit forms of the operators around the paged cache: head norms with rotation, beam selection."""
import numpy as np

import _kv_ref as ref


def norm_rotate(x, w, positions, f, magnitude, interleaved, eps):
    """x [tokens, heads, dim] float64 -> y, n (the normed head), r."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    return ref.rotate(n * w, positions, f, magnitude, interleaved), n, r


def norm_rotate_back(x, w, dy, positions, f, magnitude, interleaved, eps):
    """Gradients dx, dw and what enters them: g (dy turned back), n, r, c."""
    _, n, r = norm_rotate(x, w, positions, f, magnitude, interleaved, eps)
    g = ref.rotate(dy, positions, f, magnitude, interleaved, True)
    c = (g * w * n).mean(-1, keepdims=True)
    return r * (g * w - n * c), (g * n).sum((0, 1)), g, n, r, c


def beam_totals(logits, scores, ended, pad):
    """[groups, beams, vocab] float64 sums; -inf where there is no candidate."""
    x, out = np.asarray(logits, np.float64), None
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        lse = top + np.log(np.exp(x - np.where(np.isfinite(top), top, 0.0)).sum(-1, keepdims=True))
        out = np.asarray(scores, np.float64)[..., None] + (x - lse)
    out[~np.isfinite(out)] = -np.inf
    out[~np.isfinite(scores)] = -np.inf
    if ended is not None:
        keep = np.where(np.isfinite(scores), scores, -np.inf)
        out[ended] = -np.inf
        out[..., pad][ended] = keep[ended]
    return out


class Pages(ref.Pages):
    """The page operations on host integers, with reordering and the pages of an eviction."""

    def reorder(self, parents):
        T, n = self.T, len(parents)
        table, refs = np.full_like(self.table, -1), np.zeros_like(self.refs)
        lengths, copies, first = np.zeros_like(self.lengths), [], {}
        for i, p in enumerate(parents):
            if p >= 0:
                first.setdefault(p, i)
        for i, p in enumerate(parents):
            if p < 0:
                continue
            table[i], lengths[i] = self.table[p], self.lengths[p]
            if lengths[i] % T and (p if parents[p] == p else first[p]) != i:
                copies.append(i)
        for i in range(n):
            for j, page in enumerate(table[i]):
                if page >= 0 and not (i in copies and j == lengths[i] // T):
                    refs[page] += 1
        free = np.nonzero(refs == 0)[0]
        if len(free) < len(copies):
            return False
        for i, f in zip(copies, free):
            j = lengths[i] // T
            self.names[f] = self.names[table[i, j]]
            table[i, j], refs[f] = f, 1
        self.table, self.lengths, self.refs = table, lengths, refs
        return True

    def evict(self, keep):
        """Sequences that are cut."""
        T, free = self.T, list(np.nonzero(self.refs == 0)[0])
        cut = [s for s in range(len(keep)) if self.lengths[s] > keep[s]]
        before = self.refs.copy()
        need = [(s, j) for s in cut for j in range(-(-keep[s] // T)) if before[self.table[s, j]] > 1]
        if len(need) > len(free):
            return None
        for (s, j), f in zip(need, free):
            self.refs[self.table[s, j]] -= 1
            self.refs[f], self.table[s, j] = 1, f
        for s in cut:
            for j in range(-(-keep[s] // T), self.table.shape[1]):
                if self.table[s, j] >= 0:
                    self.refs[self.table[s, j]] -= 1
                    self.table[s, j] = -1
            self.lengths[s] = keep[s]
        return cut


def weigh(q, lse, k, n, window, scale, group):
    """q [n][Hq][D], lse [n][Hq], k [L][H][D] float64 -> weight [H][L], and the largest sum |q k| |scale| and |q . k scale|
    and |lse| that a weight came from."""
    L, H = k.shape[:2]
    out, most, top = np.zeros((H, L)), 0.0, 0.0
    for i in range(n):
        p = L - n + i
        lo, hi = (max(0, p - window + 1) if window else 0), p + 1
        if hi <= lo:
            continue
        for h in range(q.shape[1]):
            kk = k[lo:hi, h // group]
            if lse[i, h] == -np.inf:
                continue
            s = scale * (kk @ q[i, h])
            most = max(most, float(np.nanmax(np.abs(kk) @ np.abs(q[i, h])) * abs(scale)))
            top = max(top, float(np.nanmax(np.abs(s))), abs(float(lse[i, h])))
            out[h // group, lo:hi] += np.exp(s - lse[i, h])
    return out, most, top


def kept(mass, length, keep, recent):
    """Places that stay, ascending."""
    recent = min(recent, keep)
    older = np.where(np.isnan(mass[:length - recent]), -np.inf, mass[:length - recent])
    nan = np.isnan(mass[:length - recent])
    order = np.lexsort((np.arange(len(older)), nan, -older))[:keep - recent]
    return np.concatenate([np.sort(order), np.arange(length - recent, length)])
