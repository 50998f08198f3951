"""Float64 oracle of the calls that grow a draft tree or run a beam search: numpy and plain loops,
one query at a time, from the definitions in include/hedgespec.h. Test infrastructure only, like the
rest of this package; it shares no code with the GPU path."""
from __future__ import annotations

import math

import numpy as np


def row_log_softmax(z: np.ndarray, T: float):
    """log softmax(z / T) in fp64, or None where the row defines no distribution (all -inf, a NaN or
    +inf logit)."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or (z == np.inf).any() or (z == -np.inf).all():
        return None
    y = z / T
    m = y.max()
    return (y - m) - math.log(np.exp(y - m).sum())


def beam_step(logits: np.ndarray, score: np.ndarray, K: int, T: float = 1.0, done=None,
              eos: int = -1):
    """logits [B][W][V] (values as fp64), score [B][W] fp32. Returns score [B][K] fp64, parent, token
    [B][K] int32 and done [B][K] uint8."""
    B, W, V = logits.shape
    out = {"score": np.full((B, K), -np.inf), "parent": np.full((B, K), -1, np.int32),
           "token": np.full((B, K), -1, np.int32), "done": np.zeros((B, K), np.uint8)}
    for b in range(B):
        s, w, z, v = [], [], [], []  # score, beam, logit and token of every continuation
        for i in range(W):
            if not np.isfinite(score[b, i]):
                continue
            if done is not None and done[b, i]:
                s.append([float(score[b, i])])
                w.append([i])
                z.append([0.0])
                v.append([eos])
                continue
            lp = row_log_softmax(logits[b, i], T)
            if lp is None:
                continue
            t = np.flatnonzero(logits[b, i] > -np.inf)
            s.append(float(score[b, i]) + lp[t])
            w.append(np.full(len(t), i))
            z.append(logits[b, i][t])
            v.append(t)
        if not s:
            continue
        s, w, z, v = (np.concatenate(x) for x in (s, w, z, v))
        # best score, then lower beam; in a beam by logit (equal scores of unequal logits are only
        # rounding), then lower token
        order = np.lexsort((v, -z, w, -s))[:K]
        n = len(order)
        out["score"][b, :n] = s[order]
        out["parent"][b, :n] = w[order]
        out["token"][b, :n] = v[order]
        for j, o in enumerate(order):
            was = done is not None and bool(done[b, int(w[o])])
            out["done"][b, j] = was or (eos >= 0 and int(v[o]) == eos)
    return out


def beam_reorder(src: np.ndarray, dst: np.ndarray, parent: np.ndarray, count=None, axis=None):
    """dst [B][K or more]... after the call, from src [B][W]... and dst as they were before it."""
    B, K = parent.shape
    W = src.shape[1]
    out = dst.copy()
    for b in range(B):
        for j in range(K):
            p = int(parent[b, j])
            if p < 0 or p >= W:
                continue
            if count is None:
                out[b, j] = src[b, p]
            else:
                n = min(max(int(count[b]), 0), src.shape[axis])
                at = (slice(None),) * (axis - 2) + (slice(0, n),)
                out[(b, j) + at] = src[(b, p) + at]
    return out


def draft_tree(score: np.ndarray, parent: np.ndarray, token: np.ndarray, M: int):
    """score, parent, token [D][B][K]; the outputs of hs_draft_tree as a dict (mask uint64)."""
    D, B, K = score.shape
    out = {"token": np.full((B, M), -1, np.int32), "parent": np.full((B, M), -1, np.int32),
           "depth": np.full((B, M), -1, np.int32), "slot": np.full((B, M), -1, np.int32),
           "score": np.full((B, M), -np.inf, np.float32), "mask": np.zeros((B, M), np.uint64),
           "cand": np.full((B, M, K), -1, np.int32), "count": np.zeros(B, np.int32)}
    for b in range(B):
        rank = {}
        for d in range(D):
            for j in range(K):
                p, s = int(parent[d, b, j]), float(score[d, b, j])
                if p < 0 or not math.isfinite(s):
                    continue
                if d > 0 and (d - 1, p) not in rank:
                    continue
                rank[d, j] = s if d == 0 else min(s, rank[d - 1, p])
        kept = sorted(sorted(rank, key=lambda n: (-rank[n], n))[:M - 1])
        number = {n: i + 1 for i, n in enumerate(kept)}
        out["depth"][b, 0], out["score"][b, 0], out["mask"][b, 0] = 0, 0.0, 1
        out["count"][b] = len(kept) + 1
        children = {}
        for (d, j), i in number.items():
            up = 0 if d == 0 else number[d - 1, int(parent[d, b, j])]
            out["token"][b, i] = token[d, b, j]
            out["parent"][b, i], out["depth"][b, i], out["slot"][b, i] = up, d + 1, j
            out["score"][b, i] = score[d, b, j]
            out["mask"][b, i] = out["mask"][b, up] | (np.uint64(1) << np.uint64(i))
            n = children.get(up, 0)
            out["cand"][b, up, n] = token[d, b, j]
            children[up] = n + 1
    return out
