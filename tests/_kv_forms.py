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
