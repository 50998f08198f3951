"""Refusals of the calls that verify a draft: the C ABI's codes before any HIP call (the pointers are fakes, never
dereferenced) and the binding's checks before the library is called."""
import ctypes

import pytest
import torch

import paper_2510_20064_amd as hs

FAKE = 1 << 40


def _verify(**kw):
    a = hs.hs_verify_args()
    v = dict(target=hs.hs_view(FAKE, 8 * 32000, 32000), drafter=hs.hs_view(), B=2, M=8, V=32000, dtype=1,
             mode=hs.SAMPLE, depth=7, temperature=1.0, token=FAKE << 1, parent=None, count=None, u=FAKE << 2,
             out_path=FAKE << 3, out_token=FAKE << 4, out_length=FAKE << 5, workspace=FAKE << 6,
             workspace_bytes=1 << 30)
    v.update(kw)
    for k, x in v.items():
        setattr(a, k, x)
    return hs.load_library().hs_verify(ctypes.byref(a), None)


def test_verify_codes():
    size = hs.load_library().hs_verify_workspace_size
    assert size(2, 8, 32000, 1, 0) > 0 and size(2, 8, 32000, 1, 1) > size(2, 8, 32000, 1, 0)
    assert size(2, 1, 32000, 1, 1) == size(2, 1, 32000, 1, 0)
    assert size(0, 8, 32000, 1, 0) == 0 and size(2, 65, 32000, 1, 0) == 0 and size(2, 8, 0, 1, 0) == 0
    assert size(2, 8, 32000, 3, 0) == 0 and size(2, 8, (1 << 20) + 1, 1, 0) == 0 and size(65536, 8, 32000, 1, 0) == 0
    assert hs.load_library().hs_verify(None, None) == 1
    for bad in ("B", "M", "V"):
        assert _verify(**{bad: 0}) == 2, bad
    assert _verify(M=65) == 8 and _verify(B=65536) == 8
    assert _verify(V=(1 << 20) + 1) == 8 and _verify(V=(1 << 19) + 1, dtype=0) == 8
    assert _verify(dtype=3) == 3 and _verify(mode=2) == 10
    assert _verify(target=hs.hs_view(None, 0, 0)) == 1
    assert _verify(target=hs.hs_view(FAKE + 2, 0, 0)) == 4
    assert _verify(target=hs.hs_view(FAKE, 8 * 32000, 32001)) == 4
    assert _verify(target=hs.hs_view(FAKE, 8 * 32000, -8)) == 2
    assert _verify(drafter=hs.hs_view(FAKE + 8, 0, 0)) == 4
    assert _verify(drafter=hs.hs_view(FAKE << 7, 7 * 32000, 32000), parent=FAKE << 8) == 6
    for need in ("token", "u", "out_path", "out_token", "out_length"):
        assert _verify(**{need: None}) == 1, need
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-31, 1e31):
        assert _verify(temperature=t) == 5, t
    assert _verify(depth=-1) == 2 and _verify(depth=8) == 2
    assert _verify(workspace=None) == 7 and _verify(workspace_bytes=100) == 7
    assert _verify(workspace=(FAKE << 6) + 8) == 4


def test_verify_overlaps():
    assert _verify(out_path=FAKE << 1) == 10                       # the tokens
    assert _verify(out_length=(FAKE << 1) + 4 * 15) == 10          # the last token
    assert _verify(parent=FAKE << 8, out_token=FAKE << 8) == 10
    assert _verify(count=FAKE << 8, out_length=FAKE << 8) == 10
    assert _verify(out_token=(FAKE << 2) + 8 * 15) == 10           # the last number
    assert _verify(out_token=(FAKE << 3) + 4) == 10                # two outputs
    assert _verify(out_path=(FAKE << 6) + 64) == 10                # the workspace
    assert _verify(workspace=FAKE + 256) == 10                     # in the logits
    assert _verify(workspace=(FAKE << 7) + 256, drafter=hs.hs_view(FAKE << 7, 7 * 32000, 32000)) == 10


def test_verify_binding_refuses():
    z = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    tok, u = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.float64)
    for kw in (dict(token=tok.long()), dict(token=tok[:, :3]), dict(u=None), dict(u=u.float()), dict(u=u[:1]),
               dict(parent=tok.long()), dict(parent=tok.T), dict(count=torch.zeros(3, dtype=torch.int32)),
               dict(drafter=z), dict(drafter=z[:, :3].float()), dict(V=65), dict(target=z[0]),
               dict(target=z.transpose(1, 2)), dict(out=dict(path=tok.float())),
               dict(out=dict(length=torch.zeros(2, 1, dtype=torch.int32))),
               dict(workspace=torch.zeros(64, 64, dtype=torch.uint8).T), {}):
        args = dict(target=z, token=tok, u=u)
        args.update(kw)
        with pytest.raises(ValueError):  # (the last: on the CPU)
            hs.Verify(**args)
    with pytest.raises(TypeError):
        hs.Verify(z.double(), tok, u)


# ---- attention and append ----------------------------------------------------------------------------------

def _cache(**kw):
    v = dict(k=FAKE, v=FAKE + (1 << 36), k_scale=FAKE + (1 << 37), v_scale=FAKE + (1 << 38), pages=100, heads=8,
             page=64, dim=128)
    v.update(kw)
    return hs.hs_cache(*[v[n] for n, _ in hs.hs_cache._fields_])


def _rows(at, n, heads, dim=128, **kw):
    v = dict(ptr=at, stride_b=n * heads * dim, stride_n=heads * dim, stride_h=dim)
    v.update(kw)
    return hs.hs_heads(*[v[x] for x, _ in hs.hs_heads._fields_])


Q, K, X, O = FAKE << 1, FAKE << 2, FAKE << 3, FAKE << 4


def _attend(**kw):
    a = hs.hs_tree_attention_args()
    v = dict(q=_rows(Q, 16, 32), k=_rows(K, 16, 8), v=_rows(X, 16, 8), out=_rows(O, 16, 32), B=2, M=16, heads=32,
             dtype=1, cache=_cache(), table=FAKE << 5, table_stride=100, slots=100, length=FAKE << 6, mask=None,
             count=None, scale=0.1, workspace=FAKE << 7, workspace_bytes=1 << 30)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return hs.load_library().hs_tree_attention(ctypes.byref(a), None)


def _append(**kw):
    a = hs.hs_cache_append_args()
    v = dict(k=_rows(K, 16, 8), v=_rows(X, 16, 8), B=2, rows=16, taken=16, dtype=1, cache=_cache(), table=FAKE << 5,
             table_stride=100, slots=100, length=FAKE << 6, path=None, path_stride=16, count=None)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return hs.load_library().hs_cache_append(ctypes.byref(a), None)


@pytest.mark.parametrize("call", [_attend, _append])
def test_cache_codes(call):
    for kw, code in ((dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1),
                     (dict(pages=0), 2), (dict(heads=0), 2), (dict(heads=257), 8), (dict(dim=288), 8),
                     (dict(dim=0), 2), (dict(dim=48), 2), (dict(page=16), 2), (dict(page=96), 2), (dict(page=512), 8),
                     (dict(pages=1 << 31), 8), (dict(k=FAKE + 8), 4), (dict(v=FAKE + 8), 4)):
        assert call(cache=_cache(**kw)) == code, kw
    for kw, code in ((dict(table=None), 1), (dict(length=None), 1), (dict(slots=0), 2), (dict(table_stride=99), 2),
                     (dict(dtype=0), 3), (dict(dtype=3), 3), (dict(B=0), 2), (dict(B=65536), 8)):
        assert call(**kw) == code, kw
    for name, at in (("k", K), ("v", X)):
        assert call(**{name: _rows(None, 16, 8)}) == 1
        assert call(**{name: _rows(at + 8, 16, 8)}) == 4
        assert call(**{name: _rows(at, 16, 8, stride_n=1028)}) == 4
        assert call(**{name: _rows(at, 16, 8, stride_h=-128)}) == 2


def test_attention_codes():
    lib = hs.load_library()
    size = lib.hs_tree_attention_workspace_size
    assert size(2, 16, 32, 8, 128, 64, 100) > 0 and size(4096, 16, 32, 8, 128, 64, 100) == 0
    assert size(2, 16, 30, 8, 128, 64, 100) == 0
    assert lib.hs_tree_attention(None, None) == 1
    assert _attend(M=0) == 2 and _attend(heads=0) == 2 and _attend(M=65) == 8 and _attend(heads=264) == 8
    assert _attend(heads=28) == 2
    for s in (float("nan"), float("inf"), 1e39):
        assert _attend(scale=s) == 10
    assert _attend(workspace=None) == 7 and _attend(workspace_bytes=256) == 7 and _attend(workspace=(FAKE << 7) + 8) == 4
    for kw in (dict(stride_n=0), dict(stride_h=64), dict(stride_b=8), dict(stride_n=128)):
        assert _attend(out=_rows(O, 16, 32, **kw)) == 2, kw
    for at in (Q, K + 128, X + 4096, FAKE + 4096, FAKE + (1 << 36), FAKE + (1 << 37), FAKE << 5, (FAKE << 6) - 16):
        assert _attend(out=_rows(at, 16, 32)) == 10, at
    assert _attend(mask=FAKE << 8, out=_rows(FAKE << 8, 16, 32)) == 10
    assert _attend(count=FAKE << 8, out=_rows(FAKE << 8, 16, 32)) == 10
    assert _attend(workspace=O + 256) == 10 and _attend(workspace=Q + 256) == 10


def test_append_codes():
    assert hs.load_library().hs_cache_append(None, None) == 1
    assert _append(rows=0) == 2 and _append(taken=0) == 2 and _append(taken=17) == 2
    assert _append(rows=(1 << 24) + 1) == 8 and _append(taken=(1 << 24) + 1) == 8
    assert _append(path=FAKE << 8, path_stride=15) == 2
    assert _append(B=65535, taken=1 << 24, rows=1 << 24, slots=1 << 20, table_stride=1 << 20) == 8
    for name in ("k", "v", "k_scale", "v_scale"):
        for at in (K, X + 128, FAKE << 5, (FAKE << 6) - 16):
            assert _append(cache=_cache(**{name: at})) == 10, (name, at)
        assert _append(path=FAKE << 8, cache=_cache(**{name: FAKE << 8})) == 10
        assert _append(count=FAKE << 8, cache=_cache(**{name: FAKE << 8})) == 10
    assert _append(cache=_cache(v=FAKE + 4096)) == 10 and _append(cache=_cache(v_scale=FAKE + (1 << 37) + 4)) == 10


def test_cache_binding_refuses():
    bf = torch.bfloat16
    cache = hs.PagedCache.empty(4, 2, 32, 64, device="cpu")
    assert [tuple(t.shape) for t in cache.tensors.values()] == [(4, 2, 32, 64), (4, 2, 64, 32), (4, 2), (4, 2)]
    k, v, sk, sv = cache.tensors.values()
    for bad in ((k.float(), v, sk, sv), (k, k, sk, sv), (k[:3], v, sk, sv), (k, v, sk.double(), sv), (k, v, sk, sv[:3]),
                (k.view(torch.uint8).transpose(2, 3), v, sk, sv), (k[0], v, sk, sv)):
        with pytest.raises(ValueError):
            hs.PagedCache(*bad)
    q, x = torch.zeros(2, 3, 4, 64, dtype=bf), torch.zeros(2, 3, 2, 64, dtype=bf)
    table, n = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(q=q[..., :32]), dict(k=x.half()), dict(v=x[:, :2]),
               dict(k=x.transpose(2, 3)), dict(table=table.long()), dict(table=table[:1]), dict(length=n.long()),
               dict(mask=torch.zeros(2, 3)), dict(mask=torch.zeros(2, 2, dtype=torch.int64)), dict(count=n[:1]),
               dict(out=q.half()), {}):
        args = dict(q=q, k=x, v=x, cache=cache, table=table, length=n)
        args.update(kw)
        with pytest.raises(ValueError):
            hs.TreeAttention(**args)
    for kw in (dict(k=x.float()), dict(k=x[0]), dict(v=x[:, :2]), dict(path=n), dict(path=table.long()),
               dict(count=n.long()), dict(table=table.T[:1]), {}):
        args = dict(cache=cache, table=table, length=n, k=x, v=x)
        args.update(kw)
        with pytest.raises(ValueError):
            hs.CacheAppend(**args)
