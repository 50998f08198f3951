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


# ---- the cache in 8 bits ---------------------------------------------------------------------------------

def e4m3_values() -> np.ndarray:
    """The 256 codes of OCP e4m3: 4 bits of exponent (bias 7), 3 of mantissa, no infinities, NaN 0x7F and 0xFF."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    x = np.where((c & 0x7F) == 0x7F, np.nan, x)
    return np.where(c >> 7, -x, x)


VALUES = e4m3_values()


def encode(x: np.ndarray) -> np.ndarray:
    """The nearest codes, ties to the even one; beyond 448 +-448; NaN and infinities NaN (0x7F)."""
    x = np.asarray(x, dtype=np.float64)
    top = VALUES[:127]  # 0 .. 448, ascending
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    hi = np.searchsorted(top, a, side="left")
    lo = np.maximum(hi - 1, 0)
    up, down = top[hi] - a, a - top[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(top[hi] == a, hi, code)
    code = code | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def least_scale(most: float) -> float:
    """The least power of two s with most <= 448 s, from 2^-40 to 2^40."""
    e = -40
    while e < 40 and most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(k, v, k_scale, v_scale, table, length, xk, xv, path=None, count=None):
    """Changes the codes k [pages][heads][page][dim], v [pages][heads][dim][page] (uint8) and the scales (fp32) in
    place. xk, xv [B][rows][heads][dim] as fp64. Divisions are fp32."""
    pages, heads, page, _ = k.shape
    B, rows = xk.shape[:2]
    taken = rows if path is None else path.shape[1]
    f32 = np.float32
    for b in range(B):
        n = taken if count is None else min(max(int(count[b]), 0), taken)
        t, done = int(length[b]), 0
        if t < 0:
            continue
        while done < n:
            slot, first = divmod(t + done, page)
            some = min(page - first, n - done)
            ids = [done + i if path is None else int(path[b, done + i]) for i in range(some)]
            done += some
            p = int(table[b, slot]) if slot < table.shape[1] else -1
            if not 0 <= p < pages:
                continue
            for c, scale, x in ((k.transpose(0, 1, 3, 2), k_scale, xk), (v, v_scale, xv)):
                for h in range(heads):  # c[p, h] is [dim][page]
                    y = np.stack([x[b, i, h] if 0 <= i < rows else np.zeros(x.shape[3]) for i in ids], 1)
                    fin = np.abs(y[np.isfinite(y)])
                    now = least_scale(float(fin.max()) if fin.size else 0.0)
                    was = scale[p, h]
                    if first:
                        now = max(now, float(was))
                        if f32(now) != was:
                            old = VALUES[c[p, h, :, :first]].astype(f32) * (was / f32(now))
                            c[p, h, :, :first] = encode(old)
                    scale[p, h] = now
                    c[p, h, :, first:first + some] = encode(y.astype(f32) / f32(now))


def attention(q, xk, xv, k, v, k_scale, v_scale, table, length, mask=None, count=None, scale=1.0):
    """q [B][M][heads][dim], xk, xv [B][M][kv][dim] as fp64; codes and scales of the cache. Returns out as fp64 (NaN in
    rows behind count), and for each the sum of softmax |value| and the largest scale * sum |q| |k|."""
    pages, kv, page, dim = k.shape
    B, M, heads = q.shape[:3]
    group = heads // kv
    out = np.full(q.shape, np.nan)
    mean, most = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        n = M if count is None else min(max(int(count[b]), 0), M)
        tokens = min(max(int(length[b]), 0), table.shape[1] * page)
        at = [(int(table[b, t // page]), t % page) for t in range(tokens)]
        at = [(p, o) for p, o in at if 0 <= p < pages]
        p, o = np.array([x[0] for x in at], int), np.array([x[1] for x in at], int)
        for h in range(kv):
            ck = VALUES[k[p, h, o]] * k_scale[p, h, None].astype(np.float64)
            cv = VALUES[v[p, h, :, o]] * v_scale[p, h, None].astype(np.float64)
            for i in range(n):
                bits = (2 << i) - 1 if mask is None else int(mask[b, i]) % (1 << 64)
                on = [j for j in range(n) if bits >> j & 1]
                kk, vv = np.concatenate([ck, xk[b, on, h]]), np.concatenate([cv, xv[b, on, h]])
                for g in range(h * group, (h + 1) * group):
                    if not len(kk):
                        out[b, i, g] = 0.0
                        continue
                    s = kk @ q[b, i, g] * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[b, i, g] = w @ vv
                    mean[b, i, g] = w @ np.abs(vv)
                    most[b, i, g] = (np.abs(kk) @ np.abs(q[b, i, g])).max() * abs(scale)
    return out, mean, most
