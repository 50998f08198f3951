"""The measured work of the operators that grow a draft tree or run a beam search, one pass per case.

A case is a dict of plain values. Its `kind` names the operator that a pass runs:

  step     BeamStep: of the W beams of each query and the V tokens that may follow each, the K best
           continuations by score + log softmax(logits / T), with finished beams carried along;
  reorder  BeamReorder: the beams' states (caches, hidden states) moved to follow their new parents,
           in place or into other tensors, with the tokens in use counted per query;
  tree     DraftTree: the M - 1 best of the nodes that D steps have grown, as a breadth-first tree with
           parents, ancestor bits and every node's kept children.

Vocabularies are those of the repository's workloads (32000 to 151936 tokens) and odd ones between; rows
are padded to whole 16-byte vectors. Beams run from 1 to 32, the continuations kept from 1 to 64 (ten for
EAGLE's tree).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_STEP = 32 * 32 * 151936  # logits of the largest step
MAX_STATE = 2_200_000_000    # bytes of the largest states
NEG = float("-inf")


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # the smallest step in use: one query, four beams, a 32000-token head in fp32; all latency
        dict(name="step_tiny_f32", kind="step", B=1, W=4, K=4, V=32000, dtype="f32", T=1.0,
             masked="none", dead=0, finished=False),
        # interactive decoding: one level of EAGLE's tree (ten beams, ten kept), a 152k-token head
        dict(name="step_single_bf16", kind="step", B=1, W=10, K=10, V=151936, dtype="bf16", T=1.0,
             masked="none", dead=0, finished=False),
        # batched beam search with twice as many candidates as beams, some beams already finished
        dict(name="step_batch_bf16", kind="step", B=64, W=8, K=16, V=128256, dtype="bf16", T=0.7,
             masked="none", dead=0, finished=True),
        # ragged on every side: odd counts, an odd vocabulary, fp16, banned tokens, dead beams
        dict(name="step_ragged_f16", kind="step", B=13, W=5, K=11, V=50257, dtype="f16", T=0.5,
             masked="inf", dead=1, finished=True),
        # the largest step: 32 queries, 32 beams, 64 kept
        dict(name="step_wide_bf16", kind="step", B=32, W=32, K=64, V=151936, dtype="bf16", T=1.0,
             masked="low", dead=0, finished=False),
        # the hidden states of one query's ten beams follow their parents: latency
        dict(name="reorder_hidden_bf16", kind="reorder", B=1, W=10, K=10, tensors=1, H=1, cap=1,
             D=4096, dtype="bf16", inplace=False, counted=False, moved=6),
        # a batch's caches in place, keys and values of four layers, each query at its own length
        dict(name="reorder_cache_bf16", kind="reorder", B=16, W=8, K=8, tensors=8, H=8, cap=1024,
             D=128, dtype="bf16", inplace=True, counted=True, moved=4),
        # odd sizes: rows that are no multiple of 16 bytes, more kept than there were beams
        dict(name="reorder_odd_f32", kind="reorder", B=7, W=5, K=9, tensors=3, H=3, cap=77, D=33,
             dtype="f32", inplace=False, counted=True, moved=4),
        # EAGLE's tree for one query: seven steps of ten beams, 60 nodes kept and the root
        dict(name="tree_single", kind="tree", D=7, B=1, K=10, W=10, M=61),
        # a batch's trees, 64 candidates a step of which 10 were grown further
        dict(name="tree_batch", kind="tree", D=8, B=256, K=64, W=10, M=64),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "step", "step", "reorder", "reorder", "tree"])
    if kind == "step":
        V = _logint(rng, 30000, 152000)
        W = _logint(rng, 1, 32)
        K = max(1, min(64, _logint(rng, 1, 3 * W)))
        B = max(1, min(_logint(rng, 1, 128), MAX_STEP // (W * V)))
        return dict(kind=kind, B=B, W=W, K=K, V=V, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    T=rng.choice([0.5, 0.7, 1.0]), masked=rng.choice(["none", "inf", "low"]),
                    dead=rng.randint(0, max(0, W // 4)), finished=rng.random() < 0.5)
    if kind == "tree":
        K = _logint(rng, 2, 64)
        return dict(kind=kind, D=rng.randint(1, 10), B=_logint(rng, 1, 256), K=K,
                    W=rng.randint(1, K), M=rng.randint(2, 64))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    inplace = rng.random() < 0.5
    W = _logint(rng, 2, 32)
    K = W if inplace else rng.randint(1, 32)
    size = 4 if dtype == "f32" else 2
    H, D = rng.choice([1, 2, 8]), rng.choice([32, 33, 64, 100, 128])
    cap, tensors = _logint(rng, 1, 4096), rng.randint(1, 8)
    B = _logint(rng, 1, 64)
    B = max(1, min(B, MAX_STATE // (max(W, K) * H * cap * D * size * tensors)))
    cap = max(1, min(cap, MAX_STATE // (B * max(W, K) * H * D * size * tensors)))
    return dict(kind=kind, B=B, W=W, K=K, tensors=tensors, H=H, cap=cap, D=D, dtype=dtype,
                inplace=inplace, counted=rng.random() < 0.7, moved=rng.randint(1, min(W, K)))


# ---- inputs ------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 29)
    return g


def _counts(case):
    """Tokens in use per query: spread over the capacity, the same set for every seed."""
    B, cap = case["B"], case["cap"]
    return [max(1, cap * (b + 1) // B) for b in range(B)]


def _prepare_step(case, g):
    B, W, K, V, T = (case[k] for k in ("B", "W", "K", "V", "T"))
    dt = DTYPES[case["dtype"]]
    ld = (V + 7) // 8 * 8
    x = torch.zeros((B, W, ld), dtype=dt, device=DEV)
    step = max(1, (1 << 28) // (W * V))
    for b in range(0, B, step):
        n = min(step, B - b)
        z = torch.randn((n, W, V), generator=g, device=DEV) * 3.0
        at = torch.randint(0, V, (n, W, 20), generator=g, device=DEV)
        z.scatter_add_(2, at, torch.full(at.shape, 8.0, device=DEV))
        x[b:b + n, :, :V] = z
    if case["masked"] != "none":  # 500 banned tokens a row
        at = torch.randint(0, V, (B, W, 500), generator=g, device=DEV)
        low = NEG if case["masked"] == "inf" else torch.finfo(dt).min
        x.scatter_(2, at, torch.full(at.shape, low, dtype=dt, device=DEV))
    # scores as a search has them: the best beam first, a few nats apart
    score = -torch.rand((B, W), generator=g, device=DEV).mul_(1.5).cumsum(1) - 4.0
    if case["dead"]:  # the last beams of each query hold nothing yet, and NaN where logits were
        score[:, W - case["dead"]:] = NEG
        x[:, W - case["dead"]:, : V // 2] = float("nan")
    done = torch.zeros((B, W), dtype=torch.uint8, device=DEV)
    if case["finished"]:
        done[:, ::3] = (torch.rand((B, (W + 2) // 3), generator=g, device=DEV) < 0.4).to(torch.uint8)
    state = dict(kind="step", x=x, V=V, K=K, T=T, score=score, done=done, eos=2)
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.BeamStep(x, score, K, V=V, temperature=T, done=done, eos=2)
    return state


def _prepare_reorder(case, g):
    B, W, K = case["B"], case["W"], case["K"]
    shape = (case["H"], case["cap"], case["D"])
    dt = DTYPES[case["dtype"]]

    def fresh(n):
        return torch.randn((B, n) + shape, generator=g, device=DEV, dtype=dt)

    src = [fresh(W) for _ in range(case["tensors"])]
    dst = src if case["inplace"] else [fresh(K) for _ in range(case["tensors"])]
    # `moved` slots of each query continue another beam, the others their own (or, past W, any)
    ids = torch.arange(K, device=DEV).expand(B, K)
    order = torch.rand((B, K), generator=g, device=DEV).argsort(1)
    other = (ids + torch.randint(1, max(2, W), (B, K), generator=g, device=DEV)) % W
    parent = torch.where((order < case["moved"]) | (ids >= W), other, ids).to(torch.int32)
    count = None
    if case["counted"]:
        n = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)
        count = n[torch.rand(B, generator=g, device=DEV).argsort()].contiguous()
    state = dict(kind="reorder", src=src, dst=dst, parent=parent, count=count)
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.BeamReorder(src, parent, count=count, axis=3,
                                       out=None if case["inplace"] else dst)
    return state


def _prepare_tree(case, g):
    D, B, K, W, M = (case[k] for k in ("D", "B", "K", "W", "M"))
    score = torch.full((D, B, K), NEG, device=DEV)
    parent = torch.full((D, B, K), -1, dtype=torch.int32, device=DEV)
    token = torch.full((D, B, K), -1, dtype=torch.int32, device=DEV)
    up = torch.zeros((B, 1), device=DEV)
    for d in range(D):
        n = up.shape[1]
        p = torch.randint(0, n, (B, K), generator=g, device=DEV)
        p = torch.minimum(p, torch.randint(0, n, (B, K), generator=g, device=DEV))  # the best have more
        s = up.gather(1, p) - torch.empty((B, K), device=DEV).exponential_(0.7, generator=g)
        s, at = s.sort(1, descending=True)
        score[d], parent[d] = s, p.gather(1, at).to(torch.int32)
        token[d] = torch.randint(0, 151936, (B, K), generator=g, device=DEV, dtype=torch.int32)
        up = s[:, :W]
    if K > 4:  # one query in eight found fewer continuations than it may keep
        few = torch.rand(B, generator=g, device=DEV) < 0.125
        score[:, few, K - 2:] = NEG
        parent[:, few, K - 2:] = -1
        token[:, few, K - 2:] = -1
    state = dict(kind="tree", score=score, parent=parent, token=token, M=M)
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.DraftTree(score, parent, token, M)
    return state


def prepare(case, seed):
    g = _generator(seed)
    make = {"step": _prepare_step, "reorder": _prepare_reorder, "tree": _prepare_tree}[case["kind"]]
    return make(case, g)


# ---- the plain forms -----------------------------------------------------------------------------

def _plain_step(x, V, K, T, score, done, eos):
    """Scores in 64 bits: two beams' candidates often lie closer than 32 bits tell apart."""
    B, W = score.shape
    z = x[:, :, :V].double()
    m = z.amax(2, keepdim=True)
    lse = m / T + ((z - m) / T).exp().sum(2, keepdim=True).log()  # NaN: no distribution
    # each beam's K best by logit, the lower token first among equals (torch.topk promises no
    # order of ties, so it ranks whole numbers, all different)
    k = min(K, V)
    bits = x[:, :, :V].float().view(torch.int32)
    sign = bits >> 31
    rank = ((bits ^ (sign & 0x7FFFFFFF)) - sign).long()
    key = (rank << 32) + (0xFFFFFFFF - torch.arange(V, device=x.device))
    token = 0xFFFFFFFF - (key.topk(k, 2).values & 0xFFFFFFFF)
    zk = z.gather(2, token)
    s0 = score.double()[:, :, None]
    live = torch.isfinite(s0) & torch.isfinite(lse) & (zk > NEG) & (done[:, :, None] == 0)
    s = torch.where(live, s0 + (zk / T - lse), NEG)
    # a finished beam continues as itself, once
    over = (done != 0) & torch.isfinite(score)
    s[:, :, 0] = torch.where(over, score.double(), s[:, :, 0])
    token[:, :, 0] = torch.where(over, eos, token[:, :, 0])
    # the query's K best, the lower beam first among equals
    flat = s.reshape(B, W * k)
    if W * k < K:
        flat = torch.nn.functional.pad(flat, (0, K - W * k), value=NEG)
        token = torch.nn.functional.pad(token.reshape(B, W * k), (0, K - W * k))
    best, at = flat.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :K], at[:, :K]
    some = best > NEG
    parent = torch.where(some, at // k, -1)
    token = torch.where(some, token.reshape(B, -1).gather(1, at), -1)
    ended = done.gather(1, parent.clamp(min=0)) != 0
    return {"score": best.float(), "parent": parent.int(), "token": token.int(),
            "done": (some & (ended | (token == eos))).to(torch.uint8)}


def _plain_reorder_one(src, dst, parent, count):
    B, K = parent.shape
    W = src.shape[1]
    moved = src[torch.arange(B, device=src.device)[:, None], parent.long().clamp(0, W - 1)]
    keep = ((parent >= 0) & (parent < W))[:, :, None, None, None]
    if count is not None:
        keep = keep & (torch.arange(src.shape[3], device=src.device)[:, None] <
                       count[:, None, None, None, None])
    dst[:, :K] = torch.where(keep, moved, dst[:, :K])
    return dst


def _plain_tree(score, parent, token, M):
    D, B, K = score.shape
    p = parent.long()
    # a node ranks no higher than its parent, so that what is kept is a tree
    eff = [torch.where((p[0] >= 0) & torch.isfinite(score[0]), score[0], NEG)]
    for d in range(1, D):
        ok = (p[d] >= 0) & torch.isfinite(score[d])
        up = eff[d - 1].gather(1, p[d].clamp(0, K - 1))
        eff.append(torch.where(ok, torch.minimum(score[d], up), NEG))
    flat = torch.stack(eff, 1).reshape(B, D * K)
    n = min(M - 1, D * K)
    best, at = flat.sort(dim=1, descending=True, stable=True)
    kept = torch.zeros_like(flat, dtype=torch.bool).scatter(1, at[:, :n], best[:, :n] > NEG)
    count = 1 + kept.sum(1)
    index = torch.where(kept, kept.long().cumsum(1), M)  # breadth first; M: not kept
    idx = index.reshape(B, D, K)
    # node index of every node's parent: 0 (the root) for the first step
    up = [torch.zeros_like(idx[:, 0])] + [idx[:, d - 1].gather(1, p[d].clamp(0, K - 1))
                                          for d in range(1, D)]
    up = torch.stack(up, 1)
    bits = [torch.where(idx[:, 0] < M, (1 << idx[:, 0].clamp(max=63)) | 1, 0)]
    for d in range(1, D):
        own_bit = 1 << idx[:, d].clamp(max=63)
        bits.append(torch.where(idx[:, d] < M,
                                bits[d - 1].gather(1, p[d].clamp(0, K - 1)) | own_bit, 0))

    def nodes(values, root, dtype):
        """[B][M] from a value of every grown node: the root's, the kept ones', -1 (mask: 0)."""
        empty = 0 if dtype == torch.int64 else -1
        o = torch.full((B, M + 1), empty, dtype=torch.int64, device=score.device)
        o.scatter_(1, index, values.reshape(B, D * K).long())
        o[:, 0] = root
        return o[:, :M].to(dtype)

    by_step = lambda v: v.transpose(0, 1)  # noqa: E731
    slot = torch.arange(K, device=score.device).expand(B, D, K)
    depth = torch.arange(1, D + 1, device=score.device)[None, :, None].expand(B, D, K)
    node_score = torch.full((B, M + 1), NEG, device=score.device)
    node_score.scatter_(1, index, by_step(score).reshape(B, D * K))
    node_score[:, 0] = 0.0
    # place of a kept node among its parent's kept children
    k3 = kept.reshape(B, D, K)
    same = (up[:, :, :, None] == up[:, :, None, :]) & k3[:, :, None, :]
    before = torch.ones((K, K), dtype=torch.bool, device=score.device).tril(-1)
    place = (same & before).sum(3)
    at = torch.where(k3, up * K + place, M * K).reshape(B, D * K)
    cand = torch.full((B, M * K + 1), -1, dtype=torch.int32, device=score.device)
    cand.scatter_(1, at, by_step(token).reshape(B, D * K))
    return {"token": nodes(by_step(token), -1, torch.int32), "parent": nodes(up, -1, torch.int32),
            "depth": nodes(depth, 0, torch.int32), "slot": nodes(slot, -1, torch.int32),
            "mask": nodes(torch.stack(bits, 1), 1, torch.int64), "score": node_score[:, :M],
            "cand": cand[:, :M * K].reshape(B, M, K), "count": count.int()}


def run(state):
    if own:
        return state["plan"].run()
    if state["kind"] == "step":
        return _plain_step(state["x"], state["V"], state["K"], state["T"], state["score"],
                           state["done"], state["eos"])
    if state["kind"] == "reorder":
        return [_plain_reorder_one(s, d, state["parent"], state["count"])
                for s, d in zip(state["src"], state["dst"])]
    return _plain_tree(state["score"], state["parent"], state["token"], state["M"])


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    if case["kind"] == "step":
        B, W, K, V = (case[k] for k in ("B", "W", "K", "V"))
        size = 4 if case["dtype"] == "f32" else 2
        logits = B * (W - case["dead"]) * V  # a dead beam's row need not be read
        # a maximum, a multiply-add, an exponential and a sum for each logit
        return {"bytes": logits * size + 5 * B * W + 13 * B * K, "flops": 5 * logits}
    if case["kind"] == "reorder":
        size = 4 if case["dtype"] == "f32" else 2
        W, K = case["W"], case["K"]
        used = sum(_counts(case)) if case["counted"] else case["B"] * case["cap"]
        row = case["H"] * case["D"] * size * case["tensors"] * used  # one beam of every query
        if case["inplace"]:  # a beam that follows itself need not move
            return {"bytes": 2 * row * case["moved"] + 4 * case["B"] * K, "flops": 0}
        return {"bytes": row * (min(W, K) + K) + 4 * case["B"] * K, "flops": 0}
    D, B, K, M = (case[k] for k in ("D", "B", "K", "M"))
    return {"bytes": 12 * D * B * K + B * (M * (28 + 4 * K) + 4), "flops": 0}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _exact_step(s):
    x, V, K, T, eos = s["x"], s["V"], s["K"], s["T"], s["eos"]
    score, done = s["score"].double(), s["done"].bool()
    B, W = score.shape
    rows = []
    for b in range(B):  # every continuation of a query, sorted at once
        z = x[b, :, :V].double()
        total = torch.log_softmax(z / T, 1) + score[b][:, None]
        total[torch.isnan(total) | ~torch.isfinite(score[b])[:, None]] = NEG
        total[done[b]] = NEG
        total[done[b], eos] = score[b][done[b]]
        top, at = total.reshape(-1).sort(descending=True, stable=True)
        top, at = top[:K], at[:K]
        some = top > NEG
        parent = torch.where(some, at // V, -1)
        token = torch.where(some, at % V, -1)
        ended = some & (done[b][parent.clamp(min=0)] | (token == eos))
        rows.append((top, parent.int(), token.int(), ended.to(torch.uint8)))
    names = ("score", "parent", "token", "done")
    return {n: torch.stack([r[i] for r in rows]) for i, n in enumerate(names)}


def _exact_reorder(s):
    parent = s["parent"].cpu().tolist()
    count = None if s["count"] is None else s["count"].cpu().tolist()
    outs = []
    for src, dst in zip(s["src"], s["dst"]):
        o = dst.double()
        for b, row in enumerate(parent):
            n = src.shape[3] if count is None else count[b]
            for j, q in enumerate(row):
                o[b, j, :, :n] = src[b, q, :, :n].double()
        outs.append(o)
    return outs


def _exact_tree(s):
    score, parent, token = (s[n].cpu().tolist() for n in ("score", "parent", "token"))
    M = s["M"]
    D, B, K = s["score"].shape
    names = ("token", "parent", "depth", "slot", "mask", "score")
    out = {n: [] for n in names + ("cand", "count")}
    for b in range(B):
        grown = {}  # (step, slot) -> effective score
        for d in range(D):
            for j in range(K):
                v, q = score[d][b][j], parent[d][b][j]
                above = 0.0 if d == 0 else grown.get((d - 1, q))
                if q >= 0 and math.isfinite(v) and above is not None:
                    grown[d, j] = v if d == 0 else min(v, above)
        best = sorted(grown, key=lambda n: (-grown[n], n))[: M - 1]
        number = {n: i + 1 for i, n in enumerate(sorted(best))}
        nodes = [(-1, -1, 0, -1, 1, 0.0)]
        children = [[] for _ in range(M)]
        for (d, j), i in sorted(number.items()):
            up = 0 if d == 0 else number[d - 1, parent[d][b][j]]
            mask = nodes[up][4] | (1 << i)
            nodes.append((token[d][b][j], up, d + 1, j, mask, score[d][b][j]))
            children[up].append(token[d][b][j])
        nodes += [(-1, -1, -1, -1, 0, NEG)] * (M - len(nodes))
        for i, n in enumerate(names):
            out[n].append([v[i] for v in nodes])
        out["mask"][-1] = [v - (1 << 64) if v >> 63 else v for v in out["mask"][-1]]
        out["cand"].append([c + [-1] * (K - len(c)) for c in children])
        out["count"].append(len(best) + 1)
    types = {"mask": torch.int64, "score": torch.float64}
    return {n: torch.tensor(v, dtype=types.get(n, torch.int32)) for n, v in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"step": _exact_step, "reorder": _exact_reorder, "tree": _exact_tree}[case["kind"]](s)
