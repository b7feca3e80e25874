"""Float64 references of the serving operators (oracle side, test infrastructure).

Rows of a drafted tree attend the cached tokens of their group and those
drafted tokens that their mask names; weights are the softmax of the seen
scores, and a row that sees nothing gives zeros.  Eviction keeps the recent
tokens and the best ranked of the others.
"""
import numpy as np


def seen_by_tree(length, masks, M):
    """Which of the length + M rows each of the M drafted tokens sees."""
    seen = np.ones((M, length + M), dtype=bool)
    for i in range(M):
        for j in range(M):
            seen[i, length + j] = (int(masks[i]) >> j) & 1
    return seen


def attend(q, K, V, seen, scale=None):
    """q [r, d], K, V [t, d], seen [r, t] -> (out [r, d], weights [r, t])."""
    q = np.asarray(q, dtype=np.float64)
    scale = 1.0 / np.sqrt(q.shape[1]) if scale is None else scale
    out = np.zeros(q.shape)
    w = np.zeros(seen.shape)
    for r in range(q.shape[0]):
        at = np.flatnonzero(seen[r])
        if at.size == 0:
            continue
        s = (K[at] @ q[r]) * scale
        p = np.exp(s - s.max())
        w[r, at] = p / p.sum()
        out[r] = w[r, at] @ V[at]
    return out, w


def kept(acc, length, keep, recent):
    """Indices of the kept tokens of one group, in order."""
    if length <= keep:
        return list(range(length))
    old = length - recent
    nan = [t for t in range(old) if np.isnan(acc[t])]
    rank = sorted((t for t in range(old) if not np.isnan(acc[t])), key=lambda t: (-acc[t], t)) + nan
    return sorted(rank[:keep - recent]) + list(range(old, length))
