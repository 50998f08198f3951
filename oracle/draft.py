"""Float64 oracle of the calls that verify a draft: numpy and plain loops, one query at a time, from the
definitions in include/hedgespec.h. Test infrastructure only, like the rest of this package; it shares no code
with the GPU path."""
from __future__ import annotations

import numpy as np


def distribution(z: np.ndarray, T: float):
    """softmax(z / T) in fp64, or None where the row defines no distribution (all -inf, a NaN or +inf logit)."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or (z == np.inf).any() or (z == -np.inf).all():
        return None
    w = np.exp((z - z.max()) / T)
    return w / w.sum()


def inverse_cdf(p: np.ndarray, u: float) -> int:
    """The first index whose running sum exceeds u times the whole; the last of any weight where rounding leaves
    none; -1 where nothing has weight."""
    some = np.flatnonzero(p > 0)
    if not len(some):
        return -1
    c = np.cumsum(p)
    v = int(np.searchsorted(c, u * c[-1], side="right"))
    return min(v, int(some[-1]))


def verify(target, token, u, parent=None, drafter=None, count=None, T=1.0, greedy=False, depth=None):
    """target [B][M][V] and drafter [B][M - 1][V] (values as fp64), token, parent [B][M], u [B][M], count [B].
    Returns path and token [B][M] and length [B]."""
    B, M, V = target.shape
    depth = M - 1 if depth is None else depth
    out = {"path": np.full((B, M), -1, np.int32), "token": np.full((B, M), -1, np.int32),
           "length": np.zeros(B, np.int32)}
    for b in range(B):
        n = M if count is None else min(max(int(count[b]), 0), M)
        up = list(range(-1, M - 1)) if parent is None else [int(x) for x in parent[b]]
        node, steps = (0 if n else None), 0
        while node is not None:
            here, node = node, None
            out["path"][b, steps] = here
            out["length"][b] = steps + 1
            p = distribution(target[b, here], T)
            kids = [c for c in range(1, n) if up[c] == here and 0 <= token[b, c] < V] if steps < depth else []
            if p is None:
                break
            if greedy:
                best = int(np.argmax(target[b, here]))
                for c in kids:
                    if node is None and int(token[b, c]) == best:
                        node = c
                out["token"][b, steps] = best
            elif drafter is None:
                left = p.copy()
                left[[int(token[b, c]) for c in kids]] = 0.0
                own = {}  # a repeated token is the first child's
                for c in kids:
                    own[c] = 0.0 if int(token[b, c]) in [int(token[b, k]) for k in own] else p[int(token[b, c])]
                for i, c in enumerate(kids):
                    if u[b, c] * (left.sum() + sum(own[k] for k in kids[i:])) < own[c]:
                        node = c
                        break
                out["token"][b, steps] = inverse_cdf(left, u[b, 0]) if node is None else token[b, node]
            else:
                for c in kids:
                    q = distribution(drafter[b, here], T)
                    x = int(token[b, c])
                    if q is not None and u[b, c] * q[x] < p[x]:
                        node = c
                    elif q is not None and np.maximum(p - q, 0).sum() > 0:
                        p = np.maximum(p - q, 0)
                out["token"][b, steps] = inverse_cdf(p, u[b, 0]) if node is None else token[b, node]
            steps += 1
    return out
