"""What the calls that verify a draft launch, and what they return where a launch fails, without a GPU: the runtime's
launch functions are stood in for by launch_recorder.cpp, in a process of their own, which executes nothing. The
pointers are fakes, never dereferenced."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
OK, ERR_HIP = 0, 9


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", lib,
                           os.path.join(HERE, "launch_recorder.cpp")])
    return lib


def ask(recorder, *calls):
    """The answers to `calls`, each (function of this file, arguments, the launch that fails)."""
    p = subprocess.run([sys.executable, os.path.abspath(__file__), recorder], input=json.dumps(calls),
                       capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr
    return json.loads(p.stdout.splitlines()[-1])


# ---- in the process that has the recorder --------------------------------------------------------------

FAKE = 1 << 40


def verify(hs, B=2, M=8, V=32000, dtype=1, depth=None, drafted=False, greedy=False):
    """(Rows that lie on each other: no pointer of a large call runs out of the address space.)"""
    a = hs.hs_verify_args()
    a.target = hs.hs_view(FAKE, 0, 0)
    if drafted:
        a.drafter = hs.hs_view(FAKE << 1, 0, 0)
    a.B, a.M, a.V, a.dtype, a.mode, a.temperature = B, M, V, dtype, hs.GREEDY if greedy else hs.SAMPLE, 1.0
    a.depth = M - 1 if depth is None else depth
    a.token, a.u, a.out_path, a.out_token, a.out_length = [FAKE << n for n in range(2, 7)]
    a.workspace = FAKE << 7
    lib = hs.load_library()
    a.workspace_bytes = lib.hs_verify_workspace_size(B, M, V, dtype, int(drafted))
    return lib.hs_verify(ctypes.byref(a), None)


def cache(hs, kv, dim, page):
    return hs.hs_cache(FAKE, FAKE + (1 << 36), FAKE + (1 << 37), FAKE + (1 << 38), 100, kv, page, dim)


def heads(hs, at, n, count, dim, still=False):
    return hs.hs_heads(at, 0 if still else n * count * dim, count * dim, dim)


def attend(hs, B=2, M=16, H=32, kv=8, dim=128, page=64, slots=100, dtype=1):
    a = hs.hs_tree_attention_args()
    a.q, a.k, a.v = [heads(hs, FAKE << n, M, c, dim) for n, c in ((1, H), (2, kv), (3, kv))]
    a.out = heads(hs, FAKE << 4, M, H, dim)
    a.B, a.M, a.heads, a.dtype, a.scale, a.cache = B, M, H, dtype, 0.1, cache(hs, kv, dim, page)
    a.table, a.table_stride, a.slots, a.length = FAKE << 5, slots, slots, FAKE << 6
    lib = hs.load_library()
    a.workspace_bytes = lib.hs_tree_attention_workspace_size(B, M, H, kv, dim, page, slots)
    a.workspace = FAKE << 7 if a.workspace_bytes else None
    return lib.hs_tree_attention(ctypes.byref(a), None)


def append(hs, B=2, rows=16, taken=16, kv=8, dim=128, page=64, slots=100, dtype=1):
    a = hs.hs_cache_append_args()
    a.k, a.v = [heads(hs, FAKE << n, rows, kv, dim, True) for n in (1, 2)]
    a.B, a.rows, a.taken, a.dtype, a.cache = B, rows, taken, dtype, cache(hs, kv, dim, page)
    a.table, a.table_stride, a.slots, a.length, a.path_stride = FAKE << 3, slots, slots, FAKE << 4, taken
    return hs.load_library().hs_cache_append(ctypes.byref(a), None)


def main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # before anything that loads the runtime
    sys.path.insert(0, ROOT)
    import paper_2510_20064_amd as hs

    out, launches = [], (ctypes.c_uint32 * (6 * 256))()
    for name, kw, fail_at in json.load(sys.stdin):
        rec.recorder_reset(fail_at)
        rc = globals()[name](hs, **kw)
        n = rec.recorder_launches(launches, 256)
        out.append(dict(rc=rc, error=hs.load_library().hs_last_error().decode(),
                        pending=rec.hipPeekAtLastError(),
                        launches=[list(launches[6 * i:6 * i + 6]) for i in range(min(n, 256))]))
    print(json.dumps(out))


# ---- the tests ---------------------------------------------------------------------------------------------

# (call, its launches): rows and walk; with a drafter what is left of its row and the draw too; a large tree's levels and
# walk; ranges and their join; a workgroup a query and head.
CALLS = [("verify", {}, 2), ("verify", dict(drafted=True), 4), ("verify", dict(greedy=True, drafted=True), 2),
         ("verify", dict(B=32, M=61, V=128256, depth=6), 8), ("verify", dict(B=32, M=61, V=128256, depth=0), 2),
         ("attend", {}, 2), ("attend", dict(slots=2), 1), ("attend", dict(B=4096), 1), ("append", {}, 1)]


def test_a_sound_call_launches_and_says_so(recorder):
    got = ask(recorder, *[(name, kw, -1) for name, kw, _ in CALLS])
    assert [a["rc"] for a in got] == [OK] * len(CALLS) and [a["error"] for a in got] == [""] * len(CALLS)
    assert [len(a["launches"]) for a in got] == [n for _, _, n in CALLS]


def test_a_failed_launch_is_an_error(recorder):
    """Whichever launch of a call fails: an error, with the runtime's word for it, and nothing launched after it."""
    calls = [(name, kw, at) for name, kw, n in CALLS for at in range(n)]
    for (name, kw, fail_at), a in zip(calls, ask(recorder, *calls)):
        assert a["rc"] == ERR_HIP, (name, kw, fail_at)
        assert len(a["launches"]) == fail_at + 1, (name, kw, fail_at)
        assert a["error"].startswith("kernel launch failed: ") and "no error" not in a["error"], a["error"]
        assert a["pending"] == 0


def test_no_launch_is_larger_than_the_runtime_takes(recorder):
    """A launch holds fewer than 2^32 threads along each of its dimensions: larger calls are several launches, which
    together have every workgroup (a wave a slice of 256 vectors; a workgroup a query, head and tile of rows; a workgroup a
    query, head and page)."""
    calls = [("verify", dict(B=65535, M=64, V=1 << 19, drafted=True), -1),
             ("verify", dict(B=65535, M=64, V=1 << 20, dtype=0), -1),
             ("verify", dict(B=65535, M=64, V=1 << 19, depth=10), -1),
             ("attend", dict(B=65535, M=64, H=256, kv=256, slots=1), -1),
             ("attend", dict(B=65535, M=64, H=256, kv=1, dim=256, slots=1 << 20), -1),
             ("append", dict(B=60000, rows=8192, taken=8192, kv=32, dim=32, page=32, slots=1 << 20), -1)]
    got = ask(recorder, *calls)
    assert got[1]["rc"] == 8  # beyond the longest row of fp32
    least = {0: 2 * 65535 * 64 * 256 / 4, 3: 65535 * 256, 4: 65535 * 64 * 256 / 128, 5: 2 * 60000 * 32 * 257}
    for i, a in enumerate(got):
        if i == 1:
            continue
        name, kw, _ = calls[i]
        assert a["rc"] == OK, (name, kw, a["error"])
        assert all(v[0] * v[3] < 1 << 32 for v in a["launches"]), (name, kw)
        if i in least:
            assert sum(v[0] * v[1] * v[2] for v in a["launches"]) >= least[i], (name, kw)
    assert len(got[2]["launches"]) == 12  # eleven levels and the walk


if __name__ == "__main__":
    main()
