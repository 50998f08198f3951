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
