"""What the calls that grow a draft tree launch, and what they return where a launch fails, without a GPU: the
runtime's launch functions are stood in for by launch_recorder.cpp, in a process of their own, which executes
nothing. The pointers are fakes, never dereferenced."""
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

FAKE = 1 << 20


def step(hs, B=2, W=8, K=8, V=151936, dtype=1, shared_rows=False):
    es = 4 if dtype == 0 else 2
    ld = (V + 7) // 8 * 8
    a = hs.hs_beam_args()
    a.logits = hs.hs_view(FAKE, 0 if shared_rows else W * ld, 0 if shared_rows else ld)
    at = FAKE + (1 if shared_rows else B * W) * ld * es // 256 * 256 + 256
    a.B, a.W, a.K, a.V, a.dtype, a.temperature, a.eos = B, W, K, V, dtype, 1.0, -1
    a.score, a.score_stride = at, W
    a.out_score = at + 4 * B * W
    a.out_parent = a.out_score + 4 * B * K
    a.out_token = a.out_parent + 4 * B * K
    a.workspace = 1 << 50
    a.workspace_bytes = hs.beam_step_workspace_size(B, W, K, V, dtype)
    return hs.load_library().hs_beam_step(ctypes.byref(a), None)


def reorder(hs, n=1, B=2, W=8, K=8, rows=1, units=64, unit=16, gap=0, inplace=False, counted=False):
    row = units * unit + gap
    stride = [rows * row * max(W, K), rows * row, row]
    size = B * stride[0]
    states = (hs.hs_state * n)()
    for i in range(n):
        src = FAKE + 2 * i * size
        dst = src if inplace else src + size
        states[i] = hs.hs_state(src, dst, *stride, *stride, rows, units, unit)
    parent = FAKE + 2 * n * size
    return hs.load_library().hs_beam_reorder(states, n, B, W, K, parent, K,
                                             parent + 4 * B * K if counted else None, None)


def tree(hs, D=7, B=2, K=10, M=61):
    a = hs.hs_tree_args(FAKE, FAKE * 2, FAKE * 3, D, B, K, M)
    return hs.load_library().hs_draft_tree(ctypes.byref(a), None)


def topl(hs, B=2, N=2, K=4, V=32000, L=4, dtype=1):
    views = (hs.hs_view * (N + 1))(*[hs.hs_view(FAKE * (i + 1) * 16, K * V, V) for i in range(N + 1)])
    lib = hs.load_library()
    return lib.hs_eval_topl(views, ctypes.cast(ctypes.byref(views, ctypes.sizeof(hs.hs_view)),
                                               ctypes.POINTER(hs.hs_view)), N, B, K, V, dtype, L, 1.0, hs.SAMPLE,
                            1 << 40, 1 << 41, 1 << 42, 1 << 50,
                            lib.hs_eval_topl_workspace_size(B, N, K, V, L, dtype), None)


def stats(hs, rows=2, V=64):
    return hs.load_library().hs_softmax_stats(FAKE, 1, rows, V, V, 1.0, FAKE << 4, FAKE << 5, FAKE << 6, None)


def stream_read(hs):
    return hs.load_library().hs_stream_read(FAKE, 4096, 4, 1, 0, FAKE << 4, None)


def play(hs):
    return hs.load_library().hs_play(FAKE, 2, 3, 0, None, FAKE << 4, None)


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

def test_a_sound_call_launches_and_says_so(recorder):
    got = ask(recorder, ("step", {}, -1), ("reorder", {}, -1), ("reorder", dict(n=33, gap=4), -1), ("tree", {}, -1))
    assert [a["rc"] for a in got] == [OK] * 4 and [a["error"] for a in got] == [""] * 4
    assert [len(a["launches"]) for a in got] == [2, 1, 2, 1]


def test_a_failed_launch_is_an_error(recorder):
    """Whichever launch of a call fails: an error, with the runtime's word for it, and nothing launched after it."""
    calls = [("step", {}, 0), ("step", {}, 1), ("reorder", {}, 0), ("reorder", dict(n=33, gap=4), 1), ("tree", {}, 0)]
    for (name, kw, fail_at), a in zip(calls, ask(recorder, *calls)):
        assert a["rc"] == ERR_HIP, (name, kw, fail_at)
        assert len(a["launches"]) == fail_at + 1, (name, kw, fail_at)
        assert a["error"].startswith("kernel launch failed: ") and "no error" not in a["error"], a["error"]
        assert a["pending"] == 0


def test_a_failed_launch_of_an_evaluation_is_an_error(recorder):
    got = ask(recorder, ("topl", {}, -1), ("stats", {}, -1), ("stream_read", {}, -1), ("play", {}, -1))
    assert [a["rc"] for a in got] == [OK] * 4 and [len(a["launches"]) for a in got] == [2, 1, 1, 1]
    calls = [("topl", {}, 0), ("topl", {}, 1), ("stats", {}, 0), ("stream_read", {}, 0), ("play", {}, 0)]
    for (name, kw, fail_at), a in zip(calls, ask(recorder, *calls)):
        assert a["rc"] == ERR_HIP and len(a["launches"]) == fail_at + 1, (name, fail_at)
        assert a["error"].startswith("kernel launch failed: ") and "no error" not in a["error"], a["error"]
        assert a["pending"] == 0


def test_no_launch_is_larger_than_the_runtime_takes(recorder):
    """A launch holds fewer than 2^32 threads along each of its dimensions: larger calls are several launches, which
    together have every workgroup (a wave a slice of two chunks of 256 vectors; a workgroup four short rows, a row of up
    to 16 KB of few slots, or 4 KB of a longer one)."""
    calls = [("step", dict(B=65535, W=64, V=1 << 20, shared_rows=True), -1),
             ("step", dict(B=65535, W=64, V=70000, shared_rows=True), -1),
             ("step", dict(B=65535, W=64, V=200, shared_rows=True), -1),
             ("reorder", dict(B=65535, W=1, K=1, rows=1030, units=1, unit=1, gap=1, counted=True), -1),
             ("reorder", dict(n=33, B=65535, W=2, K=2, rows=30, units=1, unit=5000, gap=4, inplace=True), -1),
             ("reorder", dict(B=1, W=1, K=1, units=1 << 37, unit=1), -1),
             ("reorder", dict(B=3, W=16, K=16, units=1 << 35, unit=1), -1),
             ("reorder", dict(n=2, B=40000, W=4, K=4, rows=500, units=5, unit=1000, gap=1, inplace=True), -1)]
    least = [65535 * 64 * 256 / 4, 65535 * 64 * 18 / 4, 65535 * 64 / 4, 65535 * 1030 / 4, 33 * 65535 * 30,
             (1 << 37) / 4096, 3 * (1 << 35) / 4096, 2 * 40000 * 500]
    for (name, kw, _), need, a in zip(calls, least, ask(recorder, *calls)):
        assert a["rc"] == OK, (name, kw, a["error"])
        work = a["launches"][:-1] if name == "step" else a["launches"]
        threads = {tuple(v[3:]) for v in work}
        assert threads == {(256, 1, 1)}, (name, kw)
        assert sum(v[0] * v[1] * v[2] for v in work) >= need, (name, kw)
        if name == "step":
            assert a["launches"][-1] == [kw["B"], 1, 1, 1024, 1, 1]


if __name__ == "__main__":
    main()
