"""The measured work of the operators that verify a draft, one pass per case.

A case is a dict of plain values. Its `kind` names the operator that a pass runs:

  verify  Verify: of a drafted chain or tree the nodes that the target accepts, from given random
          numbers, and the token that the target draws behind them;
  attend  TreeAttention: the drafted nodes' queries over a paged cache held in 8 bits, with a scale for
          each page and head, and over the nodes of the draft that are on their path;
  append  CacheAppend: the keys and values of the accepted nodes (or of a prompt) to that cache.

Vocabularies are those of the repository's workloads (32000 to 151936 tokens) and odd ones between; rows
are padded to whole 16-byte vectors. Drafts are chains of up to 16 tokens and trees of up to 64 nodes, the
root among them. Heads have 64, 128 or 256 dimensions, one to eight queries' heads share a cached one, and
pages hold 32 to 256 tokens.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NEG = float("-inf")
MAX_LOGITS = 64 * 17 * 151936  # of the largest verification
MAX_TOKENS = 32 * 16384        # cached tokens of 8 heads of 128 of the largest attention
MAX_ROWS = 8 * 8192            # appended rows of 8 heads of 128
FINEST, COARSEST = 2.0 ** -40, 2.0 ** 40  # the cache's scales
TOP = 448.0                    # the largest value of 8 bits (e4m3)


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # the smallest verification in use: one query, a chain of four drafted tokens, fp32; all latency
        dict(name="verify_chain_tiny_f32", kind="verify", B=1, M=5, V=32000, dtype="f32", T=1.0,
             tree=False, depth=4, masked="none", ragged=False),
        # interactive decoding: EAGLE's tree of 60 nodes and the root, seven steps deep
        dict(name="verify_tree_single_bf16", kind="verify", B=1, M=61, V=151936, dtype="bf16", T=1.0,
             tree=True, depth=7, masked="none", ragged=False),
        # odd on every side: odd counts, an odd vocabulary, fp16, banned tokens, ragged drafts
        dict(name="verify_chain_ragged_f16", kind="verify", B=13, M=7, V=50257, dtype="f16", T=0.7,
             tree=False, depth=6, masked="inf", ragged=True),
        # batched serving with chains of eight drafted tokens
        dict(name="verify_chain_batch_bf16", kind="verify", B=64, M=9, V=151936, dtype="bf16", T=1.0,
             tree=False, depth=8, masked="low", ragged=False),
        # batched serving with trees: few of the rows are on the accepted path
        dict(name="verify_tree_batch_bf16", kind="verify", B=32, M=61, V=128256, dtype="bf16", T=0.7,
             tree=True, depth=7, masked="none", ragged=True),
        # one query, one token, a short cache: latency
        dict(name="attend_token_bf16", kind="attend", B=1, M=1, heads=32, kv=8, dim=128, page=64,
             most=512, dtype="bf16", tree=False, ragged=False),
        # one query's tree over a long conversation
        dict(name="attend_tree_single_bf16", kind="attend", B=1, M=61, heads=32, kv=8, dim=128, page=64,
             most=16384, dtype="bf16", tree=True, ragged=False),
        # odd: some caches empty or ending inside a page, three heads, drafts of different sizes
        dict(name="attend_ragged_f16", kind="attend", B=7, M=13, heads=15, kv=3, dim=64, page=32,
             most=1999, dtype="f16", tree=True, ragged=True),
        # single tokens of a batch over long caches: the cache's bytes
        dict(name="attend_batch_bf16", kind="attend", B=32, M=1, heads=32, kv=8, dim=128, page=128,
             most=16384, dtype="bf16", tree=False, ragged=True),
        # trees of a batch: as much arithmetic as bytes
        dict(name="attend_tree_batch_bf16", kind="attend", B=32, M=61, heads=32, kv=8, dim=128, page=64,
             most=8192, dtype="bf16", tree=True, ragged=True),
        # the accepted path of one round of a small batch: latency
        dict(name="append_path_bf16", kind="append", B=8, rows=61, taken=5, kv=8, dim=128, page=64,
             most=8192, dtype="bf16"),
        # prompts
        dict(name="append_prompt_f16", kind="append", B=8, rows=8192, taken=8192, kv=8, dim=128, page=128,
             most=0, dtype="f16"),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "attend", "attend", "append"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "verify":
        tree = rng.random() < 0.5
        V = _logint(rng, 30000, 152000)
        M = _logint(rng, 4, 64) if tree else _logint(rng, 2, 17)
        B = max(1, min(_logint(rng, 1, 128), MAX_LOGITS // (V * (M if tree else 2 * M - 1))))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if dtype == "f32":
            B = (B + 1) // 2
        return dict(kind=kind, B=B, M=M, V=V, dtype=dtype, T=rng.choice([0.5, 0.7, 1.0]), tree=tree,
                    depth=min(M - 1, rng.randint(2, 10)) if tree else M - 1,
                    masked=rng.choice(["none", "inf", "low"]), ragged=rng.random() < 0.5)
    dim, page = rng.choice([64, 128, 128, 256]), rng.choice([32, 64, 128, 256])
    kv = rng.choice([1, 2, 3, 4, 8])
    size = kv * dim
    if kind == "attend":
        group = rng.choice([1, 2, 4, 5, 8])
        tree = rng.random() < 0.6
        M = _logint(rng, 2, 64) if tree else rng.choice([1, 1, 1, 2, 5, 9])
        most = _logint(rng, 1, 32768)
        B = _logint(rng, 1, 64)
        # neither more bytes nor more arithmetic than the largest listed cases
        B = max(1, min(B, MAX_TOKENS * 1024 // (size * most),
                       32 * 8192 * 1024 * 4 * 61 // (size * group * M * most)))
        most = max(1, min(most, MAX_TOKENS * 1024 // (size * B), 32 * 8192 * 1024 * 4 * 61 // (size * group * M * B)))
        return dict(kind=kind, B=B, M=M, heads=kv * group, kv=kv, dim=dim, page=page, most=most, dtype=dtype,
                    tree=tree, ragged=rng.random() < 0.6)
    if rng.random() < 0.5:  # the accepted nodes of a draft
        rows = _logint(rng, 1, 64)
        return dict(kind=kind, B=_logint(rng, 1, 64), rows=rows, taken=rng.randint(1, min(rows, 12)), kv=kv, dim=dim,
                    page=page, most=_logint(rng, 1, 8192), dtype=dtype)
    rows = _logint(rng, 64, 8192)
    B = max(1, min(_logint(rng, 1, 64), MAX_ROWS * 1024 // (rows * size)))
    rows = max(1, min(rows, MAX_ROWS * 1024 // (B * size)))
    return dict(kind=kind, B=B, rows=rows, taken=rows, kv=kv, dim=dim, page=page,
                most=rng.choice([0, _logint(rng, 1, 4096)]), dtype=dtype)


# ---- inputs ------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 31)
    return g


def _drafts(B, M, tree, depth, ragged, g):
    """parent [B][M], depth [B][M], ancestor bits [B][M] and count [B] (None: all M) of drafts whose nodes are
    numbered by their depth; those past the count are -1, -1 and 0."""
    at = torch.arange(M, device=DEV)
    parent = (at - 1).expand(B, M).clone()
    far = at.expand(B, M).clone()
    if tree:
        # of each step's nodes the first ones have the most children
        step = (1 + (at - 1).clamp(min=0) * depth // max(1, M - 1)).clamp(max=depth)
        step[0] = 0
        far = step.expand(B, M).clone()
        first = torch.searchsorted(step, step - 1)
        wide = torch.searchsorted(step, step) - first
        r = torch.rand((B, M), generator=g, device=DEV) * torch.rand((B, M), generator=g, device=DEV)
        parent = first + (r * wide).long()
        parent[:, 0] = -1
    count = None
    if ragged:
        count = torch.randint((M + 1) // 2, M + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        gone = at[None] >= count[:, None]
        parent[gone], far[gone] = -1, -1
    bits = torch.zeros((B, M), dtype=torch.int64, device=DEV)
    rows = torch.arange(B, device=DEV)
    for n in range(M):
        up = parent[:, n]
        above = torch.where(up >= 0, bits[rows, up.clamp(min=0)], 0)
        bits[:, n] = torch.where((up >= 0) | (n == 0), above | (1 << n), 0)
    return parent.to(torch.int32).contiguous(), far, bits, count


def _prepare_verify(case, g):
    B, M, V, T = (case[k] for k in ("B", "M", "V", "T"))
    dt = DTYPES[case["dtype"]]
    ld = (V + 7) // 8 * 8
    tree = case["tree"]
    parent, _, _, count = _drafts(B, M, tree, case["depth"], case["ragged"], g)
    target = torch.zeros((B, M, ld), dtype=dt, device=DEV)
    drafter = None if tree else torch.zeros((B, M - 1, ld), dtype=dt, device=DEV)
    token = torch.full((B, M), -1, dtype=torch.int32, device=DEV)
    low = NEG if case["masked"] == "inf" else torch.finfo(dt).min
    for b in range(B):
        z = torch.randn((M, V), generator=g, device=DEV) * 3.0
        at = torch.randint(0, V, (M, 20), generator=g, device=DEV)
        z.scatter_add_(1, at, 10.0 + 4.0 * torch.randn(at.shape, generator=g, device=DEV))
        if case["masked"] != "none":  # 500 banned tokens a row
            at = torch.randint(0, V, (M, 500), generator=g, device=DEV)
            z.scatter_(1, at, torch.full(at.shape, low, device=DEV))
        target[b, :, :V] = z
        if tree:
            # a node's children are tokens that a drafter ranks high: mostly the target's, in nearly its order
            mine = (z + 0.7 * torch.randn((M, V), generator=g, device=DEV)).topk(min(M, V), 1).indices
            up = parent[b].long()
            same = (up[:, None] == up[None, :]) & (up[None, :] >= 0)
            place = same.tril(-1).sum(1)
            token[b] = torch.where(up >= 0, mine[up.clamp(min=0), place.clamp(max=mine.shape[1] - 1)], -1)
        else:
            q = z[:-1] + 0.7 * torch.randn((M - 1, V), generator=g, device=DEV)
            drafter[b, :, :V] = q
            pick = torch.rand((M - 1, V), generator=g, device=DEV).clamp_(min=1e-30).log_().neg_().log_().neg_()
            token[b, 1:] = (drafter[b, :, :V].float() / T + pick).argmax(1)
    u = torch.rand((B, M), generator=g, device=DEV, dtype=torch.float64)
    state = dict(kind="verify", target=target, drafter=drafter, token=token, parent=parent if tree else None,
                 count=count, u=u, V=V, T=T, depth=case["depth"])
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.Verify(target, token, u, parent=state["parent"], drafter=drafter, count=count, V=V,
                                  temperature=T, depth=case["depth"])
    return state


def _lengths(case):
    """Cached tokens of each query: spread over the range, or all the most; the same set for every seed."""
    B, most = case["B"], case["most"]
    return [most * b // max(1, B - 1) if case.get("ragged") and B > 1 else most for b in range(B)]


def _codes(shape, g):
    """Values of 8 bits as a cache holds them: normal ones, the page's largest near the top of the range."""
    x = torch.empty(shape, dtype=torch.float8_e4m3fn, device=DEV)
    flat = x.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = (torch.randn(n, generator=g, device=DEV) * 90.0).clamp_(-TOP, TOP).to(x.dtype)
    return x


def _cache(case, room, g):
    """A pool of pages, and a table that gives every query the pages of its `room` tokens in any order."""
    B, kv, dim, page = (case[k] for k in ("B", "kv", "dim", "page"))
    each = max(1, -(-room // page))
    pages = B * each + 3
    k = _codes((pages, kv, page, dim), g)
    v = _codes((pages, kv, dim, page), g)
    scale = [torch.exp2(torch.randint(-8, -5, (pages, kv), generator=g, device=DEV).float()) for _ in range(2)]
    order = torch.randperm(pages, generator=g, device=DEV)[: B * each]
    return k, v, scale[0], scale[1], order.reshape(B, each).to(torch.int32).contiguous()


def _prepare_attend(case, g):
    B, M, heads, kv, dim = (case[k] for k in ("B", "M", "heads", "kv", "dim"))
    dt = DTYPES[case["dtype"]]
    ck, cv, sk, sv, table = _cache(case, case["most"], g)
    _, _, bits, count = _drafts(B, M, case["tree"], max(1, min(M - 1, 7)), case["ragged"] and M > 1, g)
    n = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    length = n[torch.rand(B, generator=g, device=DEV).argsort()].contiguous()
    # queries, keys and values of the nodes as one projection leaves them
    qkv = torch.randn((B, M, heads + 2 * kv, dim), generator=g, device=DEV).to(dt)
    out = torch.zeros((B, M, heads, dim), dtype=dt, device=DEV)
    state = dict(kind="attend", q=qkv[:, :, :heads], k=qkv[:, :, heads:heads + kv], v=qkv[:, :, heads + kv:],
                 ck=ck, cv=cv, sk=sk, sv=sv, table=table, length=length,
                 mask=bits if case["tree"] else None, count=count, scale=2.0 / math.sqrt(dim), out=out)
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.TreeAttention(state["q"], state["k"], state["v"], hs.PagedCache(ck, cv, sk, sv), table,
                                         length, mask=state["mask"], count=count, scale=state["scale"], out=out)
    return state


def _prepare_append(case, g):
    B, kv, dim, rows, taken = (case[k] for k in ("B", "kv", "dim", "rows", "taken"))
    dt = DTYPES[case["dtype"]]
    ck, cv, sk, sv, table = _cache(case, case["most"] + taken, g)
    most = case["most"]
    length = torch.randint(0, most + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    count = torch.randint((taken + 1) // 2, taken + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    path = None
    if taken < rows:  # the accepted nodes of a tree, in order
        path = torch.rand((B, rows), generator=g, device=DEV).argsort(1)[:, :taken].sort(1).values
        path = path.to(torch.int32).contiguous()
    spread = 0.5 + torch.rand((B, rows, 1, 1), generator=g, device=DEV)
    x = [(torch.randn((B, rows, kv, dim), generator=g, device=DEV) * spread * 2.0).to(dt) for _ in range(2)]
    state = dict(kind="append", k=x[0], v=x[1], ck=ck, cv=cv, sk=sk, sv=sv, table=table, length=length,
                 path=path, count=count)
    if own:
        import paper_2510_20064_amd as hs

        state["plan"] = hs.CacheAppend(hs.PagedCache(ck, cv, sk, sv), table, length, x[0], x[1], path=path,
                                       count=count)
    return state


def prepare(case, seed):
    g = _generator(seed)
    make = {"verify": _prepare_verify, "attend": _prepare_attend, "append": _prepare_append}[case["kind"]]
    return make(case, g)


# ---- the plain forms -----------------------------------------------------------------------------

def _weights(z, T):
    """exp((z - max) / T) of rows in 64 bits, 0 for a row that defines no distribution, and which do."""
    z = z.double()
    m = z.amax(1, keepdim=True)
    ok = torch.isfinite(m)
    return torch.where(ok, ((z - torch.where(ok, m, 0.0)) / T).exp(), 0.0), ok[:, 0]


def _pick(w, total, u):
    """The first token whose running sum of w exceeds u total; the last of any weight where rounding leaves none."""
    over = w.cumsum(1) > (u * total)[:, None]
    last = w.shape[1] - 1 - (w > 0).flip(1).to(torch.uint8).argmax(1)
    return torch.where(over.any(1), torch.minimum(over.to(torch.uint8).argmax(1), last), last)


def _plain_verify(s):
    """In 64 bits: a random number next to the border of two tokens decides between them."""
    V, T, u, count = s["V"], s["T"], s["u"], s["count"]
    target, drafter = s["target"][:, :, :V], s["drafter"]
    B, M, _ = target.shape
    rows = torch.arange(B, device=DEV)
    at = torch.arange(M, device=DEV)
    n = torch.full((B,), M, device=DEV) if count is None else count.long()
    parent = (at - 1).expand(B, M) if s["parent"] is None else s["parent"].long()
    token = s["token"].long()
    sound = (at[None] < n[:, None]) & (at[None] > 0) & (token >= 0) & (token < V)
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    walking = n > 0
    path = torch.full((B, M), -1, dtype=torch.long, device=DEV)
    emitted = torch.full((B, M), -1, dtype=torch.long, device=DEV)
    length = torch.zeros(B, dtype=torch.long, device=DEV)
    for step in range(s["depth"] + 1):
        path[:, step] = torch.where(walking, cur, path[:, step])
        w, ok = _weights(target[rows, cur], T)
        child = sound & (parent == cur[:, None]) & (step < s["depth"])
        x = torch.where(child, token, 0)
        if drafter is None:
            twice = ((x[:, :, None] == x[:, None, :]) & child[:, None, :]).tril(-1).any(2)
            mine = torch.where(child & ~twice, w.gather(1, x), 0.0)
            w = torch.cat([w, w[:, :1]], 1).scatter(1, torch.where(child, x, V), 0.0)[:, :V]
            total = w.sum(1)
            left = total[:, None] + mine.flip(1).cumsum(1).flip(1)
            takes = u * left < mine
        else:
            p = w / w.sum(1, keepdim=True).clamp(min=1e-300)
            f, fine = _weights(drafter[rows, cur.clamp(max=M - 2), :V], T)
            q = f / f.sum(1, keepdim=True).clamp(min=1e-300)
            some = child.any(1)
            takes = child & fine[:, None] & (u * q.gather(1, x) < p.gather(1, x))
            rest = (p - q).clamp(min=0)
            w = torch.where((some & (rest.sum(1) > 0))[:, None], rest, p)
            total = w.sum(1)
        takes = takes & child & ok[:, None]
        goes = takes.any(1)
        to = takes.to(torch.uint8).argmax(1)
        drawn = torch.where(ok, _pick(w, total, u[:, 0]), -1)
        emitted[:, step] = torch.where(walking, torch.where(goes, token[rows, to], drawn), emitted[:, step])
        length += walking
        walking = walking & goes
        cur = torch.where(walking, to, cur)
    return {"path": path.int(), "token": emitted.int(), "length": length.int()}


def _paged(c, scale, table, last):
    """[B][kv][tokens][dim] fp32 of the pages of every query; last: a page holds its tokens last."""
    x = c[table.long()].float() * scale[table.long()][:, :, :, None, None]
    x = x.transpose(3, 4) if last else x
    B, each, kv, page, dim = x.shape
    return x.transpose(1, 2).reshape(B, kv, each * page, dim)


def _plain_attend(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    B, M, heads, dim = q.shape
    kv = k.shape[2]
    ck, cv = _paged(s["ck"], s["sk"], s["table"], False), _paged(s["cv"], s["sv"], s["table"], True)
    cached = torch.arange(ck.shape[2], device=DEV)[None] < s["length"][:, None]
    at = torch.arange(M, device=DEV)
    n = torch.full((B,), M, device=DEV) if s["count"] is None else s["count"].long()
    bits = ((2 << at) - 1).expand(B, M) if s["mask"] is None else s["mask"]
    sees = ((bits[:, :, None] >> at) & 1).bool() & (at < n[:, None])[:, None, :]
    sees = torch.cat([cached[:, None].expand(B, M, cached.shape[1]), sees], 2)  # [B][M][tokens]
    keys = torch.cat([ck, k.transpose(1, 2)], 2)
    values = torch.cat([cv.masked_fill(~cached[:, None, :, None], 0.0), v.transpose(1, 2)], 2)
    rows = q.reshape(B, M, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(B, kv, -1, dim)
    x = (rows @ keys.transpose(2, 3)) * s["scale"]
    x = x.reshape(B, kv, heads // kv, M, -1).masked_fill_(~sees[:, None, None], NEG)
    m = x.amax(4, keepdim=True)
    p = (x - torch.where(m > NEG, m, 0.0)).exp_()
    total = p.sum(4, keepdim=True)
    o = p.reshape(B, kv, -1, p.shape[4]) @ values
    o = o.reshape(B, kv, heads // kv, M, dim) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, M, heads, dim).to(s["out"].dtype)
    s["out"].copy_(torch.where((at < n[:, None])[:, :, None, None], o, s["out"]))
    return s["out"]


def _least_scale(most):
    """The least power of two s with most <= 448 s, in the cache's range."""
    mantissa, e = torch.frexp(most.double() / TOP)
    e = torch.where(mantissa == 0.5, e - 1, e).double()
    return torch.where(most > 0, torch.exp2(e), FINEST).clamp(FINEST, COARSEST).float()


def _plain_append_one(x, cache, scale, last, s):
    """x [B][rows][kv][dim] to a pool whose pages hold their tokens last, or before the dims."""
    table, length, path = s["table"].long(), s["length"].long(), s["path"]
    page = cache.shape[3] if last else cache.shape[2]
    B, rows = x.shape[:2]
    most = rows if path is None else path.shape[1]
    span = -(-most // page) + 1  # pages that the new rows can touch
    at = torch.arange(span * page, device=DEV)
    start = length // page
    i = at[None] - (length - start * page)[:, None]  # which of the new rows a place takes
    new = (i >= 0) & (i < s["count"].long()[:, None])
    row = i.clamp(0, most - 1)
    row = row if path is None else path.long().gather(1, row)
    y = x.float()[torch.arange(B, device=DEV)[:, None], row]  # [B][span * page][kv][dim]
    y = y.reshape(B, span, page, *x.shape[2:]).permute(0, 1, 3, 2, 4)  # [B][span][kv][page][dim]
    new = new.reshape(B, span, 1, page, 1)
    old = (i < 0).reshape(B, span, 1, page, 1)
    slot = start[:, None] + torch.arange(span, device=DEV)
    ids = table.gather(1, slot.clamp(max=table.shape[1] - 1))
    need = _least_scale(torch.where(new, y.abs(), 0.0).amax((3, 4)))
    was = scale[ids]
    held = old.any(3)[..., 0]
    now = torch.where(held, torch.maximum(need, was), need)
    kept = cache[ids].float()
    kept = kept.transpose(3, 4) if last else kept
    kept = kept * (was / now)[..., None, None]
    codes = torch.where(new, y / now[..., None, None], kept).clamp(-TOP, TOP)
    codes = torch.where(new | old, codes.to(cache.dtype).float(),
                        (cache[ids].transpose(3, 4) if last else cache[ids]).float()).to(cache.dtype)
    codes = codes.transpose(3, 4) if last else codes
    touched = new.any(3).reshape(B, span) & (slot < table.shape[1])
    cache.view(torch.uint8)[ids[touched]] = codes[touched].view(torch.uint8)
    scale[ids[touched]] = now[touched]


def run(state):
    if own:
        return state["plan"].run()
    if state["kind"] == "verify":
        return _plain_verify(state)
    if state["kind"] == "attend":
        return _plain_attend(state)
    _plain_append_one(state["k"], state["ck"], state["sk"], False, state)
    _plain_append_one(state["v"], state["cv"], state["sv"], True, state)
    return {"k": state["ck"], "v": state["cv"], "k_scale": state["sk"], "v_scale": state["sv"]}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    if case["kind"] == "verify":
        B, M, V, tree = (case[k] for k in ("B", "M", "V", "tree"))
        size = 4 if case["dtype"] == "f32" else 2
        # the rows on the accepted path: of these inputs a node's children hold the next one 77 times in 100, and 86 of
        # 100 drafted tokens of a chain are accepted; a chain's drafter has as many rows
        on = 0.77 if tree else 0.86
        rows = (1 - on ** (case["depth"] + 1)) / (1 - on) * (1 if tree else 2)
        # a maximum, a multiply-add, an exponential and a sum for each logit
        return {"bytes": int(B * (rows * V * size + M * 24)), "flops": int(5 * B * rows * V)}
    B, kv, dim, page = (case[k] for k in ("B", "kv", "dim", "page"))
    if case["kind"] == "attend":
        M, heads, tokens = case["M"], case["heads"], sum(_lengths(case))
        return {"bytes": 2 * tokens * kv * dim + 8 * kv * (tokens // page) + 2 * B * M * dim * (2 * heads + 2 * kv),
                "flops": 4 * M * heads * dim * tokens}
    taken = 0.75 * case["taken"]  # half of them to all
    return {"bytes": int(2 * B * taken * kv * dim * 3), "flops": int(4 * B * taken * kv * dim)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _distribution(z, T):
    z = z.double().cpu()
    if bool(torch.isnan(z).any()) or float(z.max()) in (math.inf, -math.inf):
        return None
    return torch.softmax(z / T, 0)


def _inverse(p, u):
    c = p.cumsum(0)
    v = int(torch.searchsorted(c, u * float(c[-1]), right=True))
    return min(v, int(p.nonzero().max()))


def _exact_verify(s):
    """Rejection by rejection: the mass left to a node's later children is what the earlier ones did not have."""
    V, T, M = s["V"], s["T"], s["target"].shape[1]
    u, token = s["u"].cpu().tolist(), s["token"].cpu().tolist()
    out = {"path": [], "token": [], "length": []}
    for b in range(len(u)):
        n = M if s["count"] is None else int(s["count"][b])
        up = list(range(-1, M - 1)) if s["parent"] is None else s["parent"][b].tolist()
        path, emitted = [], []
        node = 0 if n else None
        while node is not None:
            path.append(node)
            p = _distribution(s["target"][b, node, :V], T)
            children = [c for c in range(1, n) if up[c] == node and 0 <= token[b][c] < V]
            children = children if len(path) <= s["depth"] else []
            if p is None:
                emitted.append(-1)
                break
            node = None
            for c in children:
                x = token[b][c]
                if s["drafter"] is None:
                    if u[b][c] < float(p[x]):
                        node = c
                        break
                    p[x] = 0.0
                    p = p / p.sum()
                else:
                    q = _distribution(s["drafter"][b, path[-1], :V], T)
                    if q is not None and u[b][c] < (float(p[x] / q[x]) if float(q[x]) > 0 else float(p[x]) * math.inf):
                        node = c
                        break
                    rest = torch.relu(p - q) if q is not None else p
                    p = rest if float(rest.sum()) > 0 else p
            emitted.append(_inverse(p, u[b][0]) if node is None else token[b][node])
        out["path"].append(path + [-1] * (M - len(path)))
        out["token"].append(emitted + [-1] * (M - len(emitted)))
        out["length"].append(len(path))
    return {name: torch.tensor(v, dtype=torch.int32) for name, v in out.items()}


def _exact_attend(s):
    B, M, heads, dim = s["q"].shape
    kv, page = s["k"].shape[2], s["ck"].shape[2]
    group = heads // kv
    out = s["out"].double()
    for b in range(B):
        n, tokens = M if s["count"] is None else int(s["count"][b]), int(s["length"][b])
        ids = s["table"][b, : -(-tokens // page)].long()
        bits = [(2 << i) - 1 for i in range(M)] if s["mask"] is None else s["mask"][b].tolist()
        sees = torch.tensor([[(bits[i] >> j) & 1 for j in range(n)] for i in range(n)], dtype=torch.bool, device=DEV)
        for h in range(kv):
            k = (s["ck"][ids, h].double() * s["sk"][ids, h].double()[:, None, None]).reshape(-1, dim)[:tokens]
            v = s["cv"][ids, h].double().transpose(1, 2) * s["sv"][ids, h].double()[:, None, None]
            v = v.reshape(-1, dim)[:tokens]
            k, v = torch.cat([k, s["k"][b, :n, h].double()]), torch.cat([v, s["v"][b, :n, h].double()])
            blocked = torch.cat([torch.zeros((n, tokens), dtype=torch.bool, device=DEV), ~sees], 1)
            for j in range(h * group, (h + 1) * group):
                x = s["q"][b, :n, j].double() @ k.T * s["scale"]
                x[blocked] = NEG
                out[b, :n, j] = torch.nan_to_num(torch.softmax(x, 1), nan=0.0) @ v
    return out


def _exact_append(s):
    """Every value before its rounding to 8 bits, in units of its page's scale."""
    out = {}
    for name, x, cache, scale in (("k", s["k"], s["ck"], s["sk"]), ("v", s["v"], s["cv"], s["sv"])):
        c, f = cache.double(), scale.double()
        c = c if name == "k" else c.transpose(2, 3)  # [pages][kv][page][dim]
        page = c.shape[2]
        for b, (n, t) in enumerate(zip(s["count"].tolist(), s["length"].tolist())):
            done = 0
            while done < n:
                slot, first = divmod(t + done, page)
                some = min(page - first, n - done)
                rows = torch.arange(done, done + some, device=DEV)
                rows = rows if s["path"] is None else s["path"][b, done:done + some].long()
                y = x[b, rows].double().transpose(0, 1)  # [kv][some][dim]
                p = int(s["table"][b, slot])
                need = torch.exp2((y.abs().amax((1, 2)) / TOP).log2().ceil()).clamp(FINEST, COARSEST)
                now = torch.maximum(need, f[p]) if first else need
                c[p, :, :first] *= (f[p] / now)[:, None, None]
                c[p, :, first:first + some] = (y / now[:, None, None]).clamp(-TOP, TOP)
                f[p] = now
                done += some
        out[name], out[name + "_scale"] = c if name == "k" else c.transpose(2, 3).contiguous(), f
    return {n: out[n] for n in ("k", "v", "k_scale", "v_scale")}


def exact(case, seed):
    s = prepare(case, seed)
    return {"verify": _exact_verify, "attend": _exact_attend, "append": _exact_append}[case["kind"]](s)
