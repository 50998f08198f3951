"""Refusals of hs_beam_step, hs_beam_reorder and hs_draft_tree: the C ABI's codes before any HIP call
(the pointers are fakes, never dereferenced) and the binding's checks before the library is called."""
import ctypes
import gc
import os
import random
import re
import weakref

import pytest
import torch

import paper_2510_20064_amd as hs

FAKE = 0x100000


def test_binding_constants_match_the_header():
    head = open(os.path.join(os.path.dirname(__file__), "..", "include", "hedgespec.h")).read()
    defs = {m.group(1): int(m.group(2)) for m in re.finditer(r"^#define (HS_\w+) (\d+)", head, re.M)}
    assert defs["HS_MAX_BEAMS"] == hs.MAX_BEAMS
    assert defs["HS_MAX_DEPTH"] == hs.MAX_DEPTH
    assert defs["HS_MAX_STATES"] == hs.MAX_STATES


def _step(**kw):
    a = hs.hs_beam_args()
    a.logits = kw.pop("logits", hs.hs_view(FAKE, 8 * 151936, 151936))
    v = dict(B=2, W=8, K=8, V=151936, dtype=1, temperature=1.0, score=FAKE << 8, done=None,
             score_stride=8, eos=2, out_score=FAKE << 9, out_parent=FAKE << 10,
             out_token=FAKE << 11, out_done=None, workspace=FAKE << 12, workspace_bytes=1 << 30)
    v.update(kw)
    for k, x in v.items():
        setattr(a, k, x)
    return hs.load_library().hs_beam_step(ctypes.byref(a), None)


def test_beam_step_codes():
    lib = hs.load_library()
    size = lib.hs_beam_step_workspace_size
    assert size(2, 8, 8, 151936, 1) > 0
    assert size(0, 8, 8, 151936, 1) == 0 and size(2, 65, 8, 151936, 1) == 0
    assert size(2, 8, 65, 151936, 1) == 0 and size(2, 8, 8, 0, 1) == 0
    assert size(2, 8, 8, 151936, 3) == 0 and size(2, 8, 8, (1 << 20) + 1, 1) == 0
    assert lib.hs_beam_step(None, None) == 1
    for bad in ("B", "W", "K", "V"):
        assert _step(**{bad: 0}) == 2, bad
    assert _step(W=65, score_stride=65) == 8
    assert _step(K=65) == 8
    assert _step(B=65536) == 8
    assert _step(V=(1 << 20) + 1) == 8
    assert _step(V=(1 << 19) + 1, dtype=0) == 8
    assert _step(dtype=3) == 3
    assert _step(logits=hs.hs_view(None, 0, 0)) == 1
    assert _step(logits=hs.hs_view(FAKE + 2, 8 * 151936, 151936)) == 4
    assert _step(logits=hs.hs_view(FAKE, 8 * 151936, 151937)) == 4
    assert _step(logits=hs.hs_view(FAKE, -8, 151936)) == 2
    for bad in ("score", "out_score", "out_parent", "out_token"):
        assert _step(**{bad: None}) == 1, bad
    assert _step(score_stride=7) == 2
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-31, 1e31):
        assert _step(temperature=t) == 5, t
    assert _step(workspace=None) == 7
    assert _step(workspace_bytes=100) == 7
    assert _step(workspace=(FAKE << 12) + 8) == 4


def test_beam_step_overlaps():
    sc = FAKE << 8
    assert _step(out_score=sc + 4) == 10                       # shifted by one beam
    assert _step(out_score=sc, K=4) == 10                      # in place with other rows
    assert _step(out_score=sc, score_stride=16) == 10
    assert _step(out_parent=sc + 60) == 10                     # the last beam of the last query
    assert _step(done=FAKE << 13, out_done=(FAKE << 13) + 1) == 10
    assert _step(done=FAKE << 13, out_token=FAKE << 13) == 10


def test_beam_step_outputs_and_workspace_apart():
    out, ws, lg = FAKE << 9, FAKE << 12, FAKE
    assert _step(out_parent=out + 60) == 10                    # the last slot of the last query
    assert _step(out_token=FAKE << 10) == 10                   # parent and token in one buffer
    assert _step(out_done=out, done=FAKE << 13) == 10
    assert _step(workspace=sc_page(out), out_score=sc_page(out) + 64) == 10
    assert _step(score=ws + 4096) == 10                        # in the workspace
    assert _step(out_score=lg + 2 * (16 * 151936) - 4) == 10   # the last logits
    assert _step(workspace=lg + 256) == 10


def sc_page(p):
    return p // 4096 * 4096


def _state(**kw):
    v = dict(src=FAKE, dst=FAKE, src_stride_b=8 * 64, src_stride_w=64, src_stride_row=0,
             dst_stride_b=8 * 64, dst_stride_w=64, dst_stride_row=0, rows=1, units=4, unit=16)
    v.update(kw)
    return hs.hs_state(*[v[n] for n, _ in hs.hs_state._fields_])


def _reorder(states, n=None, B=2, W=8, K=8, parent=FAKE << 8, stride=8, count=None):
    arr = (hs.hs_state * max(1, len(states)))(*states)
    return hs.load_library().hs_beam_reorder(arr if states else None, len(states) if n is None else n,
                                             B, W, K, parent, stride, count, None)


def test_beam_reorder_codes():
    ok = _state()
    assert _reorder([], n=1) == 1
    assert _reorder([ok], parent=None) == 1
    assert _reorder([ok], n=0) == 2
    for bad in ("B", "W", "K"):
        assert _reorder([ok], **{bad: 0}) == 2, bad
    assert _reorder([ok], W=65) == 8
    assert _reorder([ok], K=65, stride=65) == 8
    assert _reorder([ok], n=hs.MAX_STATES + 1) == 8
    assert _reorder([ok], stride=7) == 2
    assert _reorder([_state(src=None)]) == 1
    assert _reorder([_state(dst=None)]) == 1
    for bad in ("rows", "units", "unit"):
        assert _reorder([_state(**{bad: 0})]) == 2, bad
    assert _reorder([_state(src_stride_w=-64)]) == 2
    assert _reorder([_state(dst_stride_b=-64)]) == 2
    assert _reorder([_state(units=1 << 40, unit=1 << 40)]) == 8
    assert _reorder([_state(units=1 << 50, unit=16, dst=1 << 60, dst_stride_w=1 << 54,
                            dst_stride_b=1 << 57)]) == 8       # more workgroups than 2^31


def test_beam_reorder_overlaps():
    far = FAKE << 4
    assert _reorder([_state(dst_stride_w=128, dst_stride_b=1024)]) == 10   # in place, other strides
    assert _reorder([_state(dst=FAKE + 64)]) == 10                         # shifted by one beam
    assert _reorder([_state(dst=FAKE + 2 * 8 * 64 - 1)]) == 10             # by the last byte
    # rows, slots or queries of dst on top of each other
    assert _reorder([_state(dst=far, dst_stride_w=48)]) == 2
    assert _reorder([_state(dst=far, dst_stride_w=0)]) == 2
    assert _reorder([_state(dst=far, dst_stride_b=64)]) == 2
    assert _reorder([_state(dst=far, rows=2, src_stride_row=64, dst_stride_row=32)]) == 2
    # into a buffer that another state of the call reads
    assert _reorder([_state(), _state(src=far, dst=FAKE)]) == 10
    assert _reorder([_state(src=far, dst=far << 4), _state(src=far << 4, dst=far << 8)]) == 10


def test_beam_reorder_writes_apart():
    far = FAKE << 4
    assert _reorder([_state(dst=far), _state(src=FAKE << 6, dst=far)]) == 10       # one dst for two
    assert _reorder([_state(dst=far), _state(src=FAKE << 6, dst=far + 1023)]) == 10
    assert _reorder([_state(), _state()]) == 10                                    # one state twice
    assert _reorder([_state()], parent=FAKE + 1020) == 10
    assert _reorder([_state()], parent=FAKE - 60) == 10
    assert _reorder([_state()], count=FAKE - 4) == 10
    # in place the beams that are only read count too: of query 0 they are query 1's slots
    assert _reorder([_state(src_stride_b=4 * 64, dst_stride_b=4 * 64)], K=4, stride=8) == 2


def _bytes_of(at, strides, counts, row):
    (sb, sw, sr), (nb, nw, nr) = strides, counts
    starts = [at + b * sb + w * sw + r * sr for b in range(nb) for w in range(nw) for r in range(nr)]
    return starts, {s + i for s in starts for i in range(row)}


@pytest.mark.parametrize("seed", range(4))
def test_beam_reorder_refuses_every_overlap(seed):
    """Small random layouts, most of them slices of one buffer: whenever two tensors of a call share a
    byte that one of them writes (found byte by byte), the call is refused. Sound calls are not made."""
    rng = random.Random(seed)
    base, asked = 1 << 20, 0

    def strides(row):
        out, step = [0, 0, 0], row * rng.randint(1, 4)
        for d in rng.sample(range(3), 3):
            out[d] = step + rng.choice([0, 0, rng.randint(0, 8)])
            step = out[d] * rng.randint(1, 4)
        return out

    while asked < 1500:
        B, W, K, unit = rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3), rng.choice([1, 2, 4])
        n, units, nr = rng.randint(1, 4), rng.randint(1, 3), rng.randint(1, 3)
        shared = strides(units * unit)
        states, reads, writes, ok = [], [], [], True
        for _ in range(n):
            row = units * unit
            ss = shared if rng.random() < 0.8 else strides(row)
            ds = shared if rng.random() < 0.8 else strides(row)
            src, dst = base + rng.randint(0, 200), base + rng.randint(0, 200)
            if rng.random() < 0.4:
                dst = src
            if dst == src:
                ds = ss
            _, r = _bytes_of(src, ss, (B, W, nr), row)
            starts, w = _bytes_of(dst, ds, (B, max(W, K) if dst == src else K, nr), row)
            ok = ok and len(w) == len(starts) * row and (dst == src or not (r & w))
            states.append(hs.hs_state(src, dst, *ss, *ds, nr, units, unit))
            reads.append(r)
            writes.append(w)
        ok = ok and not any(i != j and writes[i] & (writes[j] | reads[j])
                            for i in range(n) for j in range(n))
        if not ok:
            asked += 1
            assert _reorder(states, B=B, W=W, K=K, parent=base - 4096, stride=4) in (2, 10)


def _tree(**kw):
    v = dict(score=FAKE, parent=FAKE, token=FAKE, D=7, B=2, K=10, M=61)
    v.update(kw)
    a = hs.hs_tree_args()
    for k, x in v.items():
        setattr(a, k, x)
    return hs.load_library().hs_draft_tree(ctypes.byref(a), None)


def test_draft_tree_codes():
    assert hs.load_library().hs_draft_tree(None, None) == 1
    for bad in ("D", "B", "K"):
        assert _tree(**{bad: 0}) == 2, bad
    assert _tree(M=1) == 2
    assert _tree(D=33) == 8
    assert _tree(K=65) == 8
    assert _tree(M=65) == 8
    assert _tree(B=65536) == 8
    for bad in ("score", "parent", "token"):
        assert _tree(**{bad: None}) == 1, bad


def test_draft_tree_outputs_apart():
    far = FAKE << 4
    last = 4 * 7 * 2 * 10
    for out, size in (("node_token", 4 * 2 * 61), ("node_mask", 8 * 2 * 61), ("cand", 4 * 2 * 61 * 10),
                      ("count", 8)):
        assert _tree(**{out: FAKE + last - 4}) == 10, out
        assert _tree(**{out: FAKE - size + 4}) == 10, out
    assert _tree(node_token=far, node_parent=far) == 10
    assert _tree(node_depth=far, node_slot=far + 4 * 2 * 61 - 4) == 10
    assert _tree(cand=far, count=far + 4 * 2 * 61 * 10 - 4) == 10


# ---- the binding: host tensors, refused before the library is called -----------------------------

def _args(B=2, W=3, V=64):
    return torch.zeros((B, W, V)), torch.zeros((B, W))


def _refused(call, words):
    with pytest.raises(ValueError, match=words):
        call()


def test_beam_step_binding_refuses():
    x, s = _args()
    _refused(lambda: hs.BeamStep(x, s, 4), "on a GPU")
    _refused(lambda: hs.BeamStep(x[0], s, 4), r"logits must be")
    _refused(lambda: hs.BeamStep(x, s, 4, V=65), "logits shape")
    _refused(lambda: hs.BeamStep(x.transpose(1, 2), torch.zeros((2, 64)), 4), "rows must be contiguous")
    _refused(lambda: hs.BeamStep(x, s.double(), 4), "score must be")
    _refused(lambda: hs.BeamStep(x, s[:, :2], 4), "score must be")
    _refused(lambda: hs.BeamStep(x, torch.zeros((3, 2)).t(), 4), "score must be")
    _refused(lambda: hs.BeamStep(x, s, 4, done=torch.zeros((2, 3))), "done must be")
    _refused(lambda: hs.BeamStep(x, s, 4, done=torch.zeros((2, 4), dtype=torch.uint8)[:, :3]),
             "done must be")
    _refused(lambda: hs.BeamStep(x, s, 4, out={"parent": torch.zeros((2, 4))}), r"out\['parent'\]")
    _refused(lambda: hs.BeamStep(x, s, 4, out={"score": torch.zeros((2, 5))}), r"out\['score'\]")
    with pytest.raises(TypeError):
        hs.BeamStep(x.double(), s, 4)


def test_beam_reorder_binding_refuses():
    x = torch.zeros((2, 3, 4, 5, 6))
    p = torch.zeros((2, 3), dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    _refused(lambda: hs.BeamReorder(x, p), "on a GPU")
    _refused(lambda: hs.BeamReorder(x, p.long()), "parent must be")
    _refused(lambda: hs.BeamReorder(x, p.t().contiguous().t()), "parent must be")
    _refused(lambda: hs.BeamReorder(x, torch.zeros((3, 3), dtype=torch.int32)), r"must be \[B\]\[W\]")
    _refused(lambda: hs.BeamReorder(x, torch.zeros((2, 4), dtype=torch.int32)), "in place K <= W")
    _refused(lambda: hs.BeamReorder(x, p, count=n), "count needs the axis")
    _refused(lambda: hs.BeamReorder(x, p, count=n.long(), axis=3), "count must be")
    _refused(lambda: hs.BeamReorder(x, p, axis=1), "axis must be")
    _refused(lambda: hs.BeamReorder(x, p, axis=5), "axis must be")
    _refused(lambda: hs.BeamReorder(x.transpose(3, 4), p), "must be contiguous")
    _refused(lambda: hs.BeamReorder(torch.zeros((2, 3, 4, 8, 6))[:, :, :, :5].transpose(2, 3), p, axis=3),
             "must be contiguous")
    _refused(lambda: hs.BeamReorder(torch.zeros((2, 3, 4, 9, 5, 6))[:, :, :, :7], p, axis=4),
             "collapse to one stride")
    _refused(lambda: hs.BeamReorder([x, torch.zeros((2, 4, 1))], p), r"must be \[B\]\[W\]")
    _refused(lambda: hs.BeamReorder(x, p, out=[]), "as many out tensors")
    _refused(lambda: hs.BeamReorder(x, p, out=x.double()), "differs in type")
    _refused(lambda: hs.BeamReorder(x, p, out=torch.zeros((2, 4, 4, 5, 6))), r"out must be")


def test_draft_tree_and_growth_binding_refuse():
    s = torch.zeros((3, 2, 4))
    i = torch.zeros((3, 2, 4), dtype=torch.int32)
    _refused(lambda: hs.DraftTree(s, i, i, 5), "on a GPU")
    _refused(lambda: hs.DraftTree(s[0], i, i, 5), r"score must be \[D\]")
    _refused(lambda: hs.DraftTree(s, i.long(), i, 5), "parent must be")
    _refused(lambda: hs.DraftTree(s, i, i[:, :, :3], 5), "token must be")
    _refused(lambda: hs.DraftTree(s, i, i, 5, out={"mask": i}), r"out\['mask'\]")
    for bad in (dict(depth=0), dict(W=5), dict(K=65), dict(M=1), dict(depth=33)):
        kw = dict(B=1, depth=3, W=2, K=4, M=5, device="cpu")
        kw.update(bad)
        _refused(lambda: hs.TreeGrowth(**kw), "need 1 <= depth")


def test_growth_keeps_what_a_captured_graph_uses(monkeypatch):
    """A tree of one row length may be in a graph while one of another is grown: no level's plan and workspace are
    given up for another's, and a length that comes again has the one it had. (Nothing is launched.)"""
    made = []

    class Step(hs.BeamStep):
        def __init__(self, *a, **kw):
            super().__init__(*a, **kw)
            made.append(weakref.ref(self))

    monkeypatch.setattr(hs, "BeamStep", Step)
    monkeypatch.setattr(hs, "_one_device", lambda *t: torch.device("cpu"))
    monkeypatch.setattr(hs, "_launch", lambda *a: None)
    growth = hs.TreeGrowth(2, 2, 3, 4, 5, device="cpu")
    for V, dt in ((64, torch.float32), (72, torch.float32), (64, torch.bfloat16), (64, torch.float32)):
        for n in (1, 3):
            growth.level(torch.zeros((2, n, V), dtype=dt))
        growth.tree()
    gc.collect()
    assert all(r() is not None for r in made)
    assert len(made) == 2 * 3 and len({r().workspace.data_ptr() for r in made}) == 6
