"""GPU parity of hs_beam_step, hs_beam_reorder, hs_draft_tree and the growth of a tree by them, against
oracle/beam.py in fp64.

Tolerances. Parents, tokens and ended marks are exact: the order is that of fp64 scores. A score is
rounded once to fp32 (2^-24 of its size) after a normaliser whose fp32 exponentials are off by at most
  2^-23 (the exponential) + 17 * 2 * 2^-24 * ln 2 (the exponent: two roundings of at most 17 bits,
  where e^-|x| |x| has its weight in a row of 2^17 logits) + 10 * 2^-24 (sums of 32)
of themselves: 2.2e-6 together if every one were off the same way.
Moved bytes and trees are exact.
"""
import numpy as np
import pytest
import torch

import paper_2510_20064_amd as hs
from oracle import beam

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NORM_TOL = 2.2e-6


def note(msg):
    print("\n[case] " + msg, flush=True)


def rows(g, B, W, V, dt, pad=8, scale=3.0):
    """[B][W][ld] logits on the GPU, ld a multiple of 8, NaN behind V."""
    ld = (V + pad - 1) // pad * pad
    x = torch.full((B, W, ld), float("nan"), dtype=dt)
    x[:, :, :V] = (torch.randn((B, W, V), generator=g) * scale).to(dt)
    return x


def scores(g, B, W):
    return -torch.rand((B, W), generator=g).cumsum(1) - 1.0


def check_step(x, score, K, V, T=1.0, done=None, eos=-1, **kw):
    out = hs.beam_step(x.cuda() if not x.is_cuda else x, score.cuda(), K, V=V, temperature=T,
                       done=None if done is None else done.cuda(), eos=eos, **kw)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    ref = beam.beam_step(x.cpu()[:, :, :V].double().numpy(), score.numpy(), K, T=T,
                         done=None if done is None else done.numpy(), eos=eos)
    same_step(got, ref)
    return got


def same_step(got, ref):
    assert np.array_equal(got["parent"], ref["parent"])
    assert np.array_equal(got["token"], ref["token"])
    if "done" in got:
        assert np.array_equal(got["done"].astype(np.uint8), ref["done"])
    some = ref["parent"] >= 0
    assert np.all(got["score"][~some] == -np.inf)
    with np.errstate(over="ignore"):
        near = np.abs(ref["score"][some]) < 1e38
    r, s = ref["score"][some][near], got["score"][some][near].astype(np.float64)
    assert np.all(np.abs(s - r) <= np.abs(r) * 2.0 ** -24 + NORM_TOL), np.abs(s - r).max()


# ---- hs_beam_step ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B,W,K,V", [(1, 1, 1, 1), (1, 1, 5, 3), (2, 3, 4, 7), (1, 64, 64, 9),
                                     (3, 1, 64, 64), (2, 4, 10, 2048), (2, 4, 10, 2049),
                                     (1, 7, 33, 4095), (3, 5, 11, 50257), (1, 2, 64, 70001)])
def test_step_sizes(dtype, B, W, K, V):
    note("step %s B=%d W=%d K=%d V=%d" % (dtype, B, W, K, V))
    g = torch.Generator().manual_seed(B * 1000 + W * 100 + K + V)
    x = rows(g, B, W, V, DTYPES[dtype])
    check_step(x, scores(g, B, W), K, V, T=0.7)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("K", [1, 10, 64])
def test_step_longest_rows(dtype, K):
    V = (1 << 19) if dtype == "f32" else (1 << 20)
    note("longest rows %s K=%d" % (dtype, K))
    g = torch.Generator().manual_seed(K)
    x = rows(g, 1, 2, V, DTYPES[dtype])
    check_step(x, scores(g, 1, 2), K, V)


@pytest.mark.parametrize("T", [1e-3, 0.25, 1.0, 1.4426950408889634, 30.0])
def test_step_temperatures(T):
    note("temperature %g" % T)
    g = torch.Generator().manual_seed(7)
    x = rows(g, 2, 3, 5000, torch.float32)
    x[:, :, 17] = float("-inf")
    check_step(x, scores(g, 2, 3), 12, 5000, T=T)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T", [1e-30, 1e-12, 1e12, 1e30])
def test_step_temperatures_at_the_limits(dtype, T):
    note("temperature %g %s" % (T, dtype))
    g = torch.Generator().manual_seed(71)
    x = rows(g, 2, 3, 5003, DTYPES[dtype])
    x[0, 1, :5003:7] = float("-inf")
    x[1, 2, :5003:5] = torch.finfo(DTYPES[dtype]).min
    check_step(x, scores(g, 2, 3), 12, 5003, T=T)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("units", [127, 128, 129, 319, 320, 321, 645])
@pytest.mark.parametrize("W", [3, 17, 33])
def test_step_borders_of_units_and_rows(dtype, units, W):
    """Rows about the lengths, and beams about the numbers, at which another kernel is taken."""
    per = 256 if dtype == "f32" else 512          # logits of a unit: 16 lanes, 4 vectors each
    V = units * per - 5
    note("borders %s W=%d V=%d" % (dtype, W, V))
    g = torch.Generator().manual_seed(units + W)
    x = rows(g, 1, W, V, DTYPES[dtype])
    x[0, W // 2, V - 1] = 40.0                    # the last logit of a row, and of the last unit
    x[0, W - 1, V - 2] = 40.0
    check_step(x, scores(g, 1, W), 12, V)


def test_step_peaked_rows_like_a_model():
    # 20 boosted tokens a row hold most of the mass; 32 beams, 64 kept
    note("peaked rows")
    g = torch.Generator().manual_seed(11)
    V = 32000
    z = torch.randn((2, 32, V), generator=g) * 3.0
    z.scatter_add_(2, torch.randint(0, V, (2, 32, 20), generator=g), torch.full((2, 32, 20), 8.0))
    check_step(z.to(torch.bfloat16), scores(g, 2, 32), 64, V)


def test_step_ties():
    # few levels of logits: ties within rows, across slices, and across identical beams
    note("ties")
    g = torch.Generator().manual_seed(13)
    V = 9000
    for dt in DTYPES.values():
        x = torch.randint(-3, 3, (2, 4, V), generator=g).to(dt)
        x[0, 1] = x[0, 0]          # identical beams of equal score: the lower beam first
        x[1, 2] = x[1, 1]
        x[1, 0, ::2] = -0.0        # signed zeros are equal
        x[1, 0, 1::2] = 0.0
        s = torch.tensor([[-1.0, -1.0, -3.0, -4.0], [-5.0, -2.0, -2.0, -9.0]])
        for K in (1, 7, 64):
            check_step(x, s, K, V)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_step_orders_that_fill_the_lists(dtype):
    # rising, falling and constant rows: many chunks bring more candidates than a list holds
    note("orders %s" % dtype)
    V = 30000
    dt = DTYPES[dtype]
    up = torch.linspace(-20, 20, V)
    x = torch.stack([up, up.flip(0), torch.full((V,), 3.0), up.abs(), -up.abs()])[None].to(dt)
    s = torch.tensor([[-1.0, -1.25, -1.5, -1.75, -2.0]])
    for K in (1, 10, 64):
        check_step(x, s, K, V)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_step_masks_and_empty_rows(dtype):
    note("masks %s" % dtype)
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(17)
    V = 5003
    x = rows(g, 3, 8, V, dt)
    low = torch.finfo(dt).min
    x[0, 0, :V] = float("-inf")                    # nothing left
    x[0, 1, :V] = float("-inf")
    x[0, 1, 4321] = 1.0                            # one token left
    x[0, 2, 100:] = float("-inf")                  # the tail masked
    x[0, 3, :4990] = float("-inf")                 # all but the tail
    x[0, 4, :V] = low                              # every logit at the lowest value
    x[0, 5, 5:V] = low
    x[0, 6, 77] = float("nan")                     # no distribution
    x[0, 7, 78] = float("inf")
    x[1, :, :V] = float("-inf")                    # a query with nothing at all
    x[2, :, :V] = low
    x[2, :, 9] = 0.0
    for K in (4, 64):
        check_step(x, scores(g, 3, 8), K, V, T=1.0)


@pytest.mark.parametrize("K", [1, 10, 64])
def test_step_every_unit_ties(K):
    # identical constant rows: every entry of every unit of every beam has the same score, so each list
    # overflows; then one score a beam, and one different token a beam
    note("every unit ties K=%d" % K)
    W, V = 64, 70000
    x = torch.full((2, W, V), 1.5, dtype=torch.bfloat16)
    s = torch.full((2, W), -2.0)
    s[1] = -torch.arange(W) * 1e-3
    got = check_step(x, s, K, V)
    assert got["parent"][0].tolist() == [0] * K and got["token"][0].tolist() == list(range(K))
    x[:, torch.arange(W), torch.arange(W) * 1000 + 77] = 2.5
    check_step(x, s, K, V)


def test_step_crowded_units():
    # a few units hold most of the best entries: more lanes of a unit than the quick way takes
    note("crowded units")
    g = torch.Generator().manual_seed(71)
    V = 40000
    for dt in DTYPES.values():
        z = torch.randn((2, 3, V), generator=g)
        z[:, :, 5000:7000] += 30.0
        z[1, :, 20000:20400] += 60.0
        for K in (1, 16, 64):
            check_step(z.to(dt), scores(g, 2, 3), K, V)
    # negative logits throughout (log-probabilities)
    z = torch.log_softmax(torch.randn((2, 3, V), generator=g) * 3, 2)
    for dt in DTYPES.values():
        check_step(z.to(dt), scores(g, 2, 3), 16, V)


@pytest.mark.parametrize("K", [1, 2])
def test_step_one_wave_finds_too_many(K):
    """Two units full of the largest logit, which one wave reads (units 0 and 16 of one row), and units
    between them whose largest lies below the bound by less than the test for reading them tells: the
    only entries are those that found no room at first."""
    note("one wave K=%d" % K)
    x = torch.zeros((1, 1, 17 * 256))
    vec = x.view(-1, 4)
    v = torch.arange(len(vec))
    unit = v // 256 * 4 + v % 64 // 16   # of fp32: the vectors of 16 lanes, in each quarter of 256
    for u in range(17):
        if u in (0, 16):
            vec[unit == u] = 1000.0
        else:
            vec[torch.nonzero(unit == u)[0, 0], 0] = 1000.0 - 5e-4
    check_step(x, torch.full((1, 1), -1.0), K, x.shape[2])


def test_step_many_queries():
    note("65535 queries")
    g = torch.Generator().manual_seed(73)
    B, W, V, K = 65535, 2, 64, 3
    x = torch.randn((B, W, V), generator=g).cuda()
    s = scores(g, B, W).cuda()
    out = hs.beam_step(x, s, K)
    total = (torch.log_softmax(x.double(), 2) + s.double()[:, :, None]).view(B, -1)
    top, at = total.topk(K + 1, 1)
    clear = (top[:, :-1] - top[:, 1:]).amin(1) > 1e-6      # no near-ties
    assert clear.float().mean() > 0.99
    assert torch.equal((at[:, :K] // V).int()[clear], out["parent"][clear])
    assert torch.equal((at[:, :K] % V).int()[clear], out["token"][clear])
    assert (out["score"].double() - top[:, :K]).abs().max() <= NORM_TOL + 20 * 2.0 ** -24


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("W,V", [(1, 700), (1, 83000), (17, 3000), (40, 1000)])
def test_step_more_queries_than_compute_units(dtype, W, V):
    note("258 queries %s W=%d V=%d" % (dtype, W, V))
    g = torch.Generator().manual_seed(W)
    check_step(rows(g, 258, W, V, DTYPES[dtype]), scores(g, 258, W), 6, V)


def test_step_offsets_past_32_bits():
    note("logits far apart")
    V, far = 3000, (1 << 32) + 4096
    g = torch.Generator().manual_seed(79)
    buf = torch.zeros((2 * far + V,), dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 2, V), (far, far, 1))   # the second query's first beam is the first's second
    z = (torch.randn((3, V), generator=g) * 3).to(torch.bfloat16)
    for i in range(3):
        buf[i * far:i * far + V] = z[i].cuda()
    s = scores(g, 2, 2)
    out = hs.beam_step(x, s.cuda(), 9)
    ref = beam.beam_step(torch.stack([z[:2], z[1:]]).double().numpy(), s.numpy(), 9)
    same_step({k: v.cpu().numpy() for k, v in out.items()}, ref)


def test_step_two_calls_at_once():
    note("two streams")
    g = torch.Generator().manual_seed(83)
    V = 60000
    x = [rows(g, 8, 8, V, torch.bfloat16) for _ in range(2)]
    s = scores(g, 8, 8)
    ref = [hs.beam_step(y.cuda(), s.cuda(), 12, V=V) for y in x]
    plans = [hs.BeamStep(y.cuda(), s.cuda(), 12, V=V) for y in x]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, st in zip(plans, streams):
            p.run(stream=st)
    torch.cuda.synchronize()
    for p, r in zip(plans, ref):
        assert all(torch.equal(p.out[k], r[k]) for k in r)


def test_step_large_logits():
    note("large logits")
    g = torch.Generator().manual_seed(19)
    x = rows(g, 1, 4, 3000, torch.float32)
    x[0, 1, :3000] += 1e6
    x[0, 2, :3000] *= 1e5
    x[0, 3, :3000] -= 1e7
    check_step(x, scores(g, 1, 4), 16, 3000)
    x[0, 3, 5] = 3e38                              # one token has it all
    x[0, 2, :3000] = 3e38                          # and these share it
    x[0, 1, :3000] = -3e38
    for K in (8, 64):
        check_step(x, scores(g, 1, 4), K, 3000)
    check_step(x, scores(g, 1, 4), 64, 3000, T=0.1)


def test_step_dead_and_finished_beams():
    note("dead and finished beams")
    g = torch.Generator().manual_seed(23)
    B, W, V = 4, 6, 1000
    x = rows(g, B, W, V, torch.bfloat16)
    s = scores(g, B, W)
    s[0, 2], s[0, 4] = float("-inf"), float("nan")
    x[0, 2, :V] = float("nan")
    s[1] = float("-inf")
    s[2, 1] = float("inf")
    done = torch.zeros((B, W), dtype=torch.uint8)
    done[0, 0] = done[0, 4] = 1                    # finished; finished and holding nothing
    done[2] = 1                                    # every beam has ended
    done[3, 5] = 1
    x[0, 0, :V] = float("nan")                     # not read
    for K in (3, 6, 20):
        check_step(x, s, K, V, done=done, eos=2)
        check_step(x, s, K, V, eos=int(x[3, 0, :V].float().argmax()))
        check_step(x, s, K, V, done=done, eos=V + 5)   # an end token that is no column
    check_step(x, s, 6, V, done=done.bool(), eos=2)


def test_step_strides_and_views():
    note("strides")
    g = torch.Generator().manual_seed(29)
    V = 3001
    big = torch.full((3, 5, 4, 3008), float("nan"), dtype=torch.float16, device="cuda")
    big[:, :, 1, :V] = (torch.randn((3, 5, V), generator=g) * 3).half().cuda()
    x = big[:, :, 1]                               # rows apart by four, queries by twenty
    s = scores(g, 3, 9)
    check_step(x, s[:, :5], 7, V)                  # a slice of wider rows of scores
    shared = big[:, :1, 1].expand(3, 5, 3008)      # one row for every beam (the root's children)
    check_step(shared, s[:, :5].contiguous(), 7, V)
    check_step(big[:1, :1, 1], s[:1, :1], 7, V)
    odd = torch.randn((1, 1, V), generator=g).cuda()  # one row needs no padding
    check_step(odd, s[:1, :1], 7, V)


def test_step_in_place_and_reused_workspace():
    note("in place")
    g = torch.Generator().manual_seed(31)
    B, W, V = 5, 6, 4000
    x = rows(g, B, W, V, torch.bfloat16)
    s, done = scores(g, B, W), torch.zeros((B, W), dtype=torch.uint8)
    done[:, 1] = 1
    sd, dd = s.cuda(), done.cuda()
    plan = hs.BeamStep(x.cuda(), sd, W, V=V, done=dd, eos=3, out={"score": sd, "done": dd})
    ws = plan.workspace
    for _ in range(3):                             # each step continues the last one's scores
        ref = beam.beam_step(x[:, :, :V].double().numpy(), sd.cpu().numpy(), W,
                             done=dd.cpu().numpy(), eos=3)
        out = plan.run()
        same_step({k: v.cpu().numpy() for k, v in out.items()}, ref)
    ws.fill_(255)                                  # scratch: whatever it holds
    a = {k: v.clone() for k, v in hs.beam_step(x.cuda(), s.cuda(), W, V=V, workspace=ws).items()}
    b = hs.beam_step(x.cuda(), s.cuda(), W, V=V, workspace=ws)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_step_leaves_what_is_not_its_own():
    note("guards")
    g = torch.Generator().manual_seed(37)
    x = rows(g, 3, 4, 2500, torch.float32).cuda()
    K = 5
    n = hs.beam_step_workspace_size(3, 4, K, 2500, hs.HS_F32)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    bufs = {k: torch.full((5, K), -77, dtype=dt, device="cuda") for k, dt in
            (("score", torch.float32), ("parent", torch.int32), ("token", torch.int32))}
    hs.beam_step(x, scores(g, 3, 4).cuda(), K, V=2500, workspace=ws[:n],
                 out={k: v[1:4] for k, v in bufs.items()})
    torch.cuda.synchronize()
    assert torch.all(ws[n:] == 0xA5)
    for v in bufs.values():
        assert torch.all(v[0] == -77) and torch.all(v[4] == -77) and not torch.any(v[1:4] == -77)


def test_step_on_another_stream_and_in_a_graph():
    note("stream and graph")
    g = torch.Generator().manual_seed(41)
    V = 20000
    x = rows(g, 2, 5, V, torch.bfloat16)
    other = rows(g, 2, 5, V, torch.bfloat16)
    s = scores(g, 2, 5)
    xd = x.cuda()
    plan = hs.BeamStep(xd, s.cuda(), 9, V=V)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plan.run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ref = beam.beam_step(x[:, :, :V].double().numpy(), s.numpy(), 9)
    same_step({k: v.cpu().numpy() for k, v in plan.out.items()}, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    for y in (other, x, other):
        xd.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        ref = beam.beam_step(y[:, :, :V].double().numpy(), s.numpy(), 9)
        same_step({k: v.cpu().numpy() for k, v in plan.out.items()}, ref)
        eager = hs.beam_step(xd, s.cuda(), 9, V=V)
        assert all(torch.equal(eager[k], plan.out[k]) for k in eager)


def test_step_same_row_same_result_wherever_it_stands():
    note("row independence")
    g = torch.Generator().manual_seed(43)
    x = rows(g, 1, 1, 40000, torch.bfloat16).expand(8, 4, -1).contiguous()
    s = torch.full((8, 4), -1.5)
    out = hs.beam_step(x.cuda(), s.cuda(), 16, V=40000)
    assert all(torch.equal(v, v[:1].expand_as(v)) for v in out.values())
    assert out["parent"][0].tolist() == [0, 1, 2, 3] * 4


@pytest.mark.parametrize("seed", range(12))
def test_step_random_shapes(seed):
    rng = np.random.default_rng(seed)
    B, W, K = int(rng.integers(1, 9)), int(rng.integers(1, 65)), int(rng.integers(1, 65))
    V = int(np.exp(rng.uniform(0, np.log(60000))))
    V = max(1, min(V, 2_000_000 // (B * W)))
    dtype = list(DTYPES)[int(rng.integers(3))]
    T = float(rng.choice([0.5, 0.7, 1.0, 1.3]))
    note("random step seed=%d B=%d W=%d K=%d V=%d %s T=%g" % (seed, B, W, K, V, dtype, T))
    g = torch.Generator().manual_seed(100 + seed)
    x = rows(g, B, W, V, DTYPES[dtype])
    ban = torch.rand((B, W, V), generator=g) < 0.3
    x[:, :, :V][ban] = float("-inf")
    done = (torch.rand((B, W), generator=g) < 0.2).to(torch.uint8)
    s = scores(g, B, W)
    s[torch.rand((B, W), generator=g) < 0.1] = float("-inf")
    check_step(x, s, K, V, T=T, done=done, eos=min(2, V - 1))


# ---- hs_beam_reorder -------------------------------------------------------------------------------

def check_reorder(states, parent, count=None, axis=None, out=None):
    """In place (out None) or into `out`; every byte of the buffers against the oracle."""
    src = [s.clone() for s in states]
    dst = src if out is None else [o.clone() for o in out]
    got = hs.beam_reorder(src, parent.cuda(), count=None if count is None else count.cuda(),
                          axis=axis, out=None if out is None else dst)
    torch.cuda.synchronize()
    for s0, d0, d, s in zip(states, states if out is None else out, got, src):
        want = beam.beam_reorder(s0.cpu().numpy(), d0.cpu().numpy(), parent.numpy(),
                                 None if count is None else count.numpy(), axis)
        assert np.array_equal(d.cpu().numpy(), want)
        if out is not None:
            assert torch.equal(s, s0)


def ints(g, shape, dtype=torch.int32):
    hi = 250 if dtype == torch.uint8 else 30000
    return torch.randint(0, hi, shape, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("W,K", [(1, 1), (4, 4), (5, 9), (9, 5), (17, 17), (32, 20), (64, 64)])
@pytest.mark.parametrize("shape", [(), (1,), (33,), (4096,), (3, 7, 5)])
def test_reorder_shapes(W, K, shape):
    note("reorder W=%d K=%d %s" % (W, K, shape))
    g = torch.Generator().manual_seed(W * 100 + K + len(shape))
    B = 3
    p = torch.randint(-1, W + 1, (B, K), generator=g, dtype=torch.int32)  # some of them no beam
    for dt in (torch.uint8, torch.int16, torch.int32, torch.float64):
        x = ints(g, (B, W) + shape, dt)
        check_reorder([x], p, out=[ints(g, (B, K) + shape, dt)])
        if K <= W:
            check_reorder([x], p)


def test_reorder_permutations_cycles_and_copies_in_place():
    note("permutations")
    g = torch.Generator().manual_seed(3)
    W = 11
    x = ints(g, (6, W, 500))
    p = torch.stack([torch.arange(W), torch.arange(W).flip(0), torch.arange(W).roll(1),
                     torch.zeros(W, dtype=torch.long), torch.full((W,), W - 1),
                     torch.randperm(W, generator=g)]).to(torch.int32)
    check_reorder([x], p)


@pytest.mark.parametrize("dtype,D", [(torch.float16, 128), (torch.int32, 33), (torch.uint8, 7)])
@pytest.mark.parametrize("inplace", [True, False])
def test_reorder_counted_caches(dtype, D, inplace):
    note("caches %s D=%d in place %s" % (dtype, D, inplace))
    g = torch.Generator().manual_seed(D)
    B, W, H, cap = 7, 5, 3, 77
    x = [ints(g, (B, W, H, cap, D), dtype) for _ in range(3)]
    p = torch.randint(0, W, (B, W), generator=g, dtype=torch.int32)
    n = torch.tensor([0, 1, 5, 76, 77, 78, -3], dtype=torch.int32)  # clamped to [0, cap]
    o = None if inplace else [ints(g, (B, W, H, cap, D), dtype) for _ in range(3)]
    check_reorder(x, p, count=n, axis=3, out=o)
    y = [t.reshape(B, W, H, cap * D) for t in x]
    check_reorder(y, p, count=n, axis=2, out=None if o is None else [t.reshape(B, W, H, cap * D) for t in o])


def test_reorder_views_and_offsets():
    # strided queries, beams and rows; a row start at every byte; the rest of the buffers untouched
    note("views")
    g = torch.Generator().manual_seed(5)
    big = ints(g, (4, 6, 3, 5, 40), torch.uint8)
    p = torch.tensor([[2, 0, 0, 1], [3, 2, 1, 0]], dtype=torch.int32)
    for off in (0, 1, 2, 4, 8, 16):
        ref = big.clone()
        x = ref[::2, 1:5, :, :3, off:off + 24]     # dims after the beams: rows of 24 bytes, 40 apart
        x = x[:, :, :, 1]                          # [2][4][3][24], one row stride
        want = big.cpu().clone()
        v = want[::2, 1:5, :, :3, off:off + 24][:, :, :, 1]
        v.copy_(torch.from_numpy(beam.beam_reorder(v.clone().numpy(), v.clone().numpy(), p.numpy(),
                                                   [20, 24], 3)))
        hs.beam_reorder(x, p.cuda(), count=torch.tensor([20, 24], dtype=torch.int32).cuda(), axis=3)
        assert torch.equal(ref.cpu(), want), off
    wide = torch.zeros((2, 10), dtype=torch.int32)  # the first beams of more slots
    wide[:, :4] = p
    y = ints(g, (2, 4, 9))
    got = hs.beam_reorder(y.clone(), wide.cuda()[:, :4])[0]
    assert np.array_equal(got.cpu().numpy(), beam.beam_reorder(y.cpu().numpy(), y.cpu().numpy(), p.numpy()))


def test_reorder_many_tensors_of_mixed_widths():
    note("many tensors")
    g = torch.Generator().manual_seed(7)
    B, W = 2, 6
    kinds = [((64,), torch.float32), ((3,), torch.float32), ((5,), torch.uint8), ((16, 8), torch.int16)]
    x = []
    for i in range(75):
        shape, dt = kinds[i % 4]
        x.append(ints(g, (B, W) + shape, dt if dt != torch.float32 else torch.int32))
    x.append(torch.zeros((B, W, 0), device="cuda"))  # nothing to move
    p = torch.randint(0, W, (B, W), generator=g, dtype=torch.int32)
    check_reorder(x, p)


@pytest.mark.parametrize("seed", range(24))
def test_reorder_random_layouts(seed):
    """Caches of any alignment: odd dims, odd lengths, odd starts, padded rows; every byte around them."""
    rng = np.random.default_rng(2000 + seed)
    g = torch.Generator().manual_seed(2000 + seed)
    dtype = [torch.uint8, torch.float16, torch.int32][seed % 3]
    B, W, H = int(rng.integers(1, 4)), int(rng.integers(1, 20)), int(rng.integers(1, 4))
    inplace = bool(rng.integers(2))
    K = W if inplace else int(rng.integers(1, 20))
    T, D = int(rng.choice([1, 2, 7, 30, 61, 130])), int(rng.choice([1, 3, 8, 33, 64, 100]))
    pad, off = int(rng.integers(0, 3)), int(rng.integers(0, 5))
    counted = bool(rng.integers(2))
    note("layout seed=%d %s B=%d W=%d K=%d H=%d T=%d D=%d pad=%d off=%d count=%d" %
         (seed, dtype, B, W, K, H, T, D, pad, off, counted))

    def cache(n, start):
        flat = ints(g, (start + B * n * H * (T + pad) * D + 3,)).to(dtype)
        return flat, flat[start:start + B * n * H * (T + pad) * D].view(B, n, H, T + pad, D)[:, :, :, :T]

    tensors = [(cache(W, off + i), None if inplace else cache(K, 2 * i + 1)) for i in range(3)]
    parent = torch.randint(-1, W + 1, (B, K), generator=g, dtype=torch.int32)
    count = torch.randint(-1, T + 2, (B,), generator=g, dtype=torch.int32) if counted else None
    want = []
    for (sf, sv), d in tensors:
        df, dv = (sf, sv) if d is None else d
        ref = df.clone()
        rv = ref[dv.storage_offset():].as_strided(dv.shape, dv.stride())
        for b in range(B):
            n = T if count is None else min(max(int(count[b]), 0), T)
            for j in range(K):
                p = int(parent[b, j])
                if 0 <= p < W:
                    rv[b, j, :, :n] = sv[b, p, :, :n]
        want.append(ref)
    kept = [sf.clone() for (sf, _), _ in tensors]
    hs.beam_reorder([sv for (_, sv), _ in tensors], parent.cuda(),
                    count=None if count is None else count.cuda(), axis=3,
                    out=None if inplace else [d[1] for _, d in tensors])
    for ((sf, _), d), ref, was in zip(tensors, want, kept):
        assert torch.equal(sf if d is None else d[0], ref)
        if d is not None:
            assert torch.equal(sf, was)


@pytest.mark.parametrize("K,moved", [(1, 1), (2, 1), (2, 2), (4, 1), (4, 3), (8, 1), (8, 2), (8, 3), (8, 4),
                                     (8, 5), (8, 8)])
@pytest.mark.parametrize("odd", [0, 1])
def test_reorder_long_rows(K, moved, odd):
    """Rows long enough that a workgroup has several pieces of each: few and many slots that move, aligned
    or not, lengths about the pieces' ends."""
    note("long rows K=%d moved=%d odd=%d" % (K, moved, odd))
    g = torch.Generator().manual_seed(K * 100 + moved * 10 + odd)
    B, H = 3, 2
    units = (1 << 20) * 3 + 4096 * 5 + 1019 - odd      # bytes of a row, 16 MB a slot in all
    step = -(-(-(-units // 4096)) // 4 // 8) * 8 * 4096  # pieces of one workgroup lie so far apart
    base = torch.randint(0, 256, (1 << 20,), generator=g, dtype=torch.uint8).cuda()
    flat = base.repeat(B * K * H * (units + 64) // (1 << 20) + 1)
    flat[: 1 << 21] ^= 0x5A
    for i in range(0, flat.numel(), 1 << 20):            # every megabyte another
        flat[i:i + 4096] += i >> 20
    x = flat[16 + odd:][:B * K * H * (units + 48 + odd)].view(B, K, H, units + 48 + odd)[..., :units]
    for off in (0, step - units, 2 * step + 1 - units, 3 * step + 1024 - units, 5 - units, 4096 + 7 - units):
        count = torch.tensor([units + off, units, units - 17], dtype=torch.int32)
        parent = torch.arange(K, dtype=torch.int32).repeat(B, 1)
        movers = torch.randperm(K, generator=g)[:moved]
        for j in movers.tolist():
            parent[:, j] = (j + 1 + torch.randint(0, max(K - 1, 1), (B,), generator=g)) % K
        want = flat.clone()
        w = want[16 + odd:][:x.numel() + (48 + odd) * B * K * H].view(B, K, H, units + 48 + odd)
        for b in range(B):
            n = int(count[b])
            w[b, :, :, :n] = x[b][parent[b].long().cuda()][:, :, :n]
        hs.beam_reorder(x, parent.cuda(), count=count.cuda(), axis=3)
        assert torch.equal(flat, want)


@pytest.mark.parametrize("K", [1, 2, 4])
def test_reorder_long_rows_into_another_buffer(K):
    note("long rows out K=%d" % K)
    g = torch.Generator().manual_seed(K)
    n = (1 << 24) + 4097
    x = torch.randint(0, 1 << 30, (2, 3, n // 4), generator=g, dtype=torch.int32).cuda()
    out = torch.full((2, K, n // 4), -1, dtype=torch.int32, device="cuda")
    parent = torch.randint(0, 3, (2, K), generator=g, dtype=torch.int32)
    parent[1, K - 1] = -1
    want = out.clone()
    for b in range(2):
        for j in range(K):
            if parent[b, j] >= 0:
                want[b, j] = x[b, int(parent[b, j])]
    kept = x.clone()
    hs.beam_reorder(x, parent.cuda(), out=out)
    assert torch.equal(out, want) and torch.equal(x, kept)


def test_reorder_slices_of_one_buffer():
    """Tensors between each other's rows: the layers of a stacked cache, keys beside values, in place
    and from one half of a buffer to the other."""
    note("reorder slices")
    g = torch.Generator().manual_seed(31)
    B, W, L, H, T, D = 2, 5, 3, 4, 7, 6
    p = torch.randint(0, W, (B, W), generator=g, dtype=torch.int32)
    n = torch.tensor([3, 7], dtype=torch.int32)
    up = p.long()[:, :, None].cuda()
    for axis, count in ((3, n), (3, None)):
        buf = ints(g, (B, W, L, H, 2, T, D), torch.int16)
        want = buf.clone()
        moved = buf[torch.arange(B, device="cuda")[:, None], up[:, :, 0]]
        for b in range(B):
            c = T if count is None else int(count[b])
            want[b, ..., :c, :] = moved[b, ..., :c, :]
        states = [buf[:, :, l, :, kv] for l in range(L) for kv in range(2)]
        hs.beam_reorder(states, p.cuda(), count=None if count is None else count.cuda(), axis=axis)
        assert torch.equal(buf, want)
    buf = ints(g, (2, B, W, L, 11))
    kept, src = buf.clone(), [buf[0, :, :, l] for l in range(L)]
    hs.beam_reorder(src, p.cuda(), out=[buf[1, :, :, l] for l in range(L)])
    assert torch.equal(buf[0], kept[0])
    assert torch.equal(buf[1], kept[0][torch.arange(B, device="cuda")[:, None], up[:, :, 0]])
    pair = ints(g, (B, W, 2, 9), torch.uint8)       # from one half of every beam to the other
    kept = pair.clone()
    hs.beam_reorder(pair[:, :, 0], p.cuda(), out=pair[:, :, 1])
    assert torch.equal(pair[:, :, 0], kept[:, :, 0])
    assert torch.equal(pair[:, :, 1], kept[:, :, 0][torch.arange(B, device="cuda")[:, None], up[:, :, 0]])
    one = ints(g, (B, W, 12))
    with pytest.raises(hs.HsError):
        hs.beam_reorder([one, one], p.cuda())


def test_reorder_offsets_past_32_bits():
    note("long caches")
    gib = 1 << 30
    x = torch.zeros((1, 3, 3 * gib + 64), dtype=torch.uint8, device="cuda")
    x[0, 0, -64:], x[0, 1, -64:], x[0, 2, -64:] = 1, 2, 3
    hs.beam_reorder(x, torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda())
    assert x[0, :, -1].tolist() == [3, 1, 2] and x[0, :, -65].tolist() == [0, 0, 0]
    n = torch.tensor([3 * gib], dtype=torch.int32).cuda() if 3 * gib < 2 ** 31 else None
    assert n is None  # a count is 32 bits: units of two bytes below
    y = x.view(torch.int16)
    c = torch.tensor([y.shape[2] - 1], dtype=torch.int32).cuda()
    hs.beam_reorder(y, torch.tensor([[1, 1, 1]], dtype=torch.int32).cuda(), count=c, axis=2)
    assert x[0, :, -3].tolist() == [1, 1, 1] and x[0, :, -1].tolist() == [3, 1, 2]


def test_reorder_on_another_stream_and_in_a_graph():
    note("reorder stream and graph")
    g = torch.Generator().manual_seed(9)
    x = ints(g, (2, 5, 700))
    p = torch.randint(0, 5, (2, 5), generator=g, dtype=torch.int32)
    buf, pd = x.clone(), p.cuda()
    plan = hs.BeamReorder(buf, pd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plan.run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = beam.beam_reorder(x.cpu().numpy(), x.cpu().numpy(), p.numpy())
    assert np.array_equal(buf.cpu().numpy(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    for _ in range(3):
        q = torch.randint(0, 5, (2, 5), generator=g, dtype=torch.int32)
        pd.copy_(q)
        want = beam.beam_reorder(buf.cpu().numpy(), buf.cpu().numpy(), q.numpy())
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(buf.cpu().numpy(), want)


# ---- hs_draft_tree -----------------------------------------------------------------------------------

def grown(rng, D, B, K, W, ties=False, empty=0.1):
    score = np.full((D, B, K), -np.inf, np.float32)
    parent = np.full((D, B, K), -1, np.int32)
    token = rng.integers(0, 151936, (D, B, K)).astype(np.int32)
    for d in range(D):
        for b in range(B):
            p = rng.integers(0, 1 if d == 0 else W, K)
            up = np.zeros(K, np.float32) if d == 0 else score[d - 1, b, p]
            step = rng.integers(0, 3, K) if ties else rng.exponential(0.7, K)
            s = (up - step).astype(np.float32)
            order = np.argsort(-np.where(np.isnan(s), -np.inf, s), kind="stable")
            score[d, b], parent[d, b] = s[order], p[order]
    hole = rng.random((D, B, K)) < empty
    score[hole] = -np.inf
    parent[hole] = -1
    token[hole] = -1
    return score, parent, token


def check_tree(score, parent, token, M):
    out = hs.draft_tree(torch.from_numpy(score).cuda(), torch.from_numpy(parent).cuda(),
                        torch.from_numpy(token).cuda(), M)
    torch.cuda.synchronize()
    ref = beam.draft_tree(score, parent, token, M)
    for k, v in out.items():
        got = v.cpu().numpy()
        assert np.array_equal(got.view(np.uint64) if k == "mask" else got, ref[k]), k


@pytest.mark.parametrize("D,K,M", [(1, 1, 2), (1, 64, 64), (7, 10, 61), (32, 64, 64), (32, 1, 64),
                                   (5, 3, 64), (6, 13, 2), (9, 40, 33)])
@pytest.mark.parametrize("ties", [False, True])
def test_tree_matches_oracle(D, K, M, ties):
    note("tree D=%d K=%d M=%d ties=%s" % (D, K, M, ties))
    rng = np.random.default_rng(D * 100 + K + M)
    check_tree(*grown(rng, D, 5, K, max(1, K // 2), ties=ties), M)


def test_tree_of_odd_scores_and_parents():
    # scores that rise along a path, NaN and infinities, parents that are empty or no slot
    note("odd trees")
    rng = np.random.default_rng(3)
    D, B, K = 6, 8, 12
    score = rng.normal(size=(D, B, K)).astype(np.float32)
    score[rng.random((D, B, K)) < 0.1] = np.nan
    score[rng.random((D, B, K)) < 0.1] = np.inf
    score[rng.random((D, B, K)) < 0.1] = -np.inf
    score[rng.random((D, B, K)) < 0.1] = -0.0
    parent = rng.integers(-2, K + 3, (D, B, K)).astype(np.int32)
    parent[:, 3] = -1                              # a query that grew nothing
    parent[0, 5] = 7                               # of the first step every parent is the root
    token = rng.integers(0, 1000, (D, B, K)).astype(np.int32)
    for M in (2, 20, 64):
        check_tree(score, parent, token, M)


@pytest.mark.parametrize("D,K", [(1, 64), (5, 20), (32, 64)])
def test_tree_of_equal_scores(D, K):
    note("equal scores D=%d K=%d" % (D, K))
    rng = np.random.default_rng(9)
    parent = rng.integers(0, K, (D, 2, K)).astype(np.int32)
    token = rng.integers(0, 1000, (D, 2, K)).astype(np.int32)
    for v in (-1.0, 0.0, -3e38):
        score = np.full((D, 2, K), v, np.float32)
        for M in (2, 30, 64):
            check_tree(score, parent, token, M)
        score[-1, :, K // 2] = np.nextafter(np.float32(v), np.float32(-np.inf))  # one below the rest
        check_tree(score, parent, token, 64)


def test_tree_outputs_are_optional_and_guarded():
    note("tree guards")
    rng = np.random.default_rng(4)
    s, p, t = (torch.from_numpy(v).cuda() for v in grown(rng, 4, 3, 9, 5))
    full = hs.draft_tree(s, p, t, 17)
    a = hs.hs_tree_args(s.data_ptr(), p.data_ptr(), t.data_ptr(), 4, 3, 9, 17)
    bits = torch.full((5, 17), -7, dtype=torch.int64, device="cuda")
    a.node_mask = bits[1:4].data_ptr()
    hs._launch(hs.load_library().hs_draft_tree, s.device, None, hs.ctypes.byref(a))
    torch.cuda.synchronize()
    assert torch.equal(bits[1:4], full["mask"]) and torch.all(bits[0] == -7) and torch.all(bits[4] == -7)


def test_tree_many_queries():
    note("65535 trees")
    rng = np.random.default_rng(8)
    B, D, K, M = 65535, 2, 3, 5
    score = -rng.random((D, B, K)).astype(np.float32)
    score[1] -= 1.0
    parent = rng.integers(0, K, (D, B, K)).astype(np.int32)
    token = rng.integers(0, 100, (D, B, K)).astype(np.int32)
    out = hs.draft_tree(*(torch.from_numpy(v).cuda() for v in (score, parent, token)), M)
    pick = np.concatenate([np.arange(50), rng.integers(0, B, 100), np.arange(B - 50, B)])
    ref = beam.draft_tree(score[:, pick], parent[:, pick], token[:, pick], M)
    for k, v in out.items():
        got = v.cpu().numpy()[pick]
        assert np.array_equal(got.view(np.uint64) if k == "mask" else got, ref[k]), k


def test_tree_in_a_graph():
    note("tree graph")
    rng = np.random.default_rng(6)
    s, p, t = (torch.from_numpy(v).cuda() for v in grown(rng, 5, 4, 8, 4))
    plan = hs.DraftTree(s, p, t, 20)
    graph = torch.cuda.CUDAGraph()
    plan.run()
    with torch.cuda.graph(graph):
        plan.run()
    for seed in range(3):
        new = grown(np.random.default_rng(seed), 5, 4, 8, 4)
        for d, v in zip((s, p, t), new):
            d.copy_(torch.from_numpy(v))
        graph.replay()
        torch.cuda.synchronize()
        ref = beam.draft_tree(*new, 20)
        for k, v in plan.out.items():
            got = v.cpu().numpy()
            assert np.array_equal(got.view(np.uint64) if k == "mask" else got, ref[k]), k


# ---- together ----------------------------------------------------------------------------------------

def test_growing_a_draft_tree_and_its_mass():
    """A drafter whose next logits depend on its hidden state grows a tree; the states follow the
    beams, the kept nodes become candidate sets, and the target's mass on them is Theorem 2's."""
    note("growth")
    g = torch.Generator().manual_seed(47)
    B, depth, W, K, M, V, C = 3, 5, 4, 12, 20, 2000, 16
    head = (torch.randn((C, V), generator=g) * 1.5).cuda()
    emb = torch.randn((V, C), generator=g).cuda()
    h0 = torch.randn((B, C), generator=g).cuda()

    def logits(hidden):
        return (hidden @ head).to(torch.bfloat16)

    def after(hidden, token):
        return torch.tanh(0.5 * hidden + emb[token.long().clamp(min=0)])

    hidden = torch.zeros((B, W, C), device="cuda")
    growth = hs.TreeGrowth(B, depth, W, K, M, states=[hidden], temperature=0.8, device="cuda")
    for _ in range(2):  # the second tree reuses every plan
        hidden[:, 0] = h0
        ref_h, ref_score, steps = h0[:, None].clone(), torch.zeros((B, 1)), []
        for d in range(depth):
            x = logits(hidden[:, :1] if d == 0 else hidden)
            assert torch.equal(x, logits(ref_h))   # the states followed their beams
            token = growth.level(x)
            ref = beam.beam_step(x.cpu().double().numpy(), ref_score.numpy(), K, T=0.8)
            same_step({"score": growth.score[d].cpu().numpy(), "parent": growth.parent[d].cpu().numpy(),
                       "token": growth.token[d].cpu().numpy()}, ref)
            steps.append(ref)
            ref_score = growth.score[d][:, :W].cpu()
            up = torch.from_numpy(ref["parent"][:, :W]).long().cuda()
            ref_h = after(ref_h[torch.arange(B, device="cuda")[:, None], up],
                          torch.from_numpy(ref["token"][:, :W]).cuda())
            if d < depth - 1:
                hidden.copy_(after(hidden, token))
        tree = growth.tree()
        want = beam.draft_tree(growth.score.cpu().numpy(), np.stack([s["parent"] for s in steps]),
                               np.stack([s["token"] for s in steps]), M)
        for k, v in tree.items():
            got = v.cpu().numpy()
            assert np.array_equal(got.view(np.uint64) if k == "mask" else got, want[k]), k
    target = (torch.randn((B, M, V), generator=g) * 3).to(torch.bfloat16).cuda()
    _, lse, _ = hs.softmax_stats(target.view(B * M, V), temperature=0.8)
    gamma = hs.candidate_mass(target, lse.view(B, M), tree["cand"][:, None], temperature=0.8)
    p = torch.softmax(target.double() / 0.8, 2).cpu().numpy()
    for b in range(B):
        for n in range(M):
            kids = want["cand"][b, n]
            mass = p[b, n, kids[kids >= 0]].sum()
            assert abs(gamma[b, 0, n].item() - mass) <= 2e-5


def test_beam_search_with_ends_and_histories():
    """A whole beam search: step, token histories and caches moved in place, ends carried, against the
    same search in fp64."""
    note("beam search")
    g = torch.Generator().manual_seed(53)
    B, W, V, steps, eos = 2, 5, 600, 12, 0
    table = torch.randn((V, V), generator=g) * 2.0
    table[:, eos] += 3.0                            # ends come often
    td = table.cuda()
    first = torch.randint(0, V, (B,), generator=g)
    hist = torch.full((B, W, steps), -1, dtype=torch.int32, device="cuda")
    score = torch.full((B, W), float("-inf"))
    score[:, 0] = 0.0                               # one live beam
    done = torch.zeros((B, W), dtype=torch.uint8)
    sd, dd = score.cuda(), done.cuda()
    last = first[:, None].expand(B, W).cuda()
    ref_hist = [[[] for _ in range(W)] for _ in range(B)]
    ref_last = first[:, None].expand(B, W).numpy()
    ref_done = done.numpy()
    for t in range(steps):
        x = td[last]
        plan = hs.BeamStep(x, sd, W, done=dd, eos=eos, out={"score": sd, "done": dd})
        ref = beam.beam_step(table.double().numpy()[ref_last], sd.cpu().numpy(), W, done=ref_done, eos=eos)
        out = plan.run()
        same_step({k: v.cpu().numpy() for k, v in out.items()}, ref)
        hs.beam_reorder(hist, out["parent"], count=torch.full((B,), t, dtype=torch.int32, device="cuda"),
                        axis=2)
        hist[:, :, t] = out["token"]
        last = out["token"].long()
        ref_hist = [[ref_hist[b][ref["parent"][b, j]] + [int(ref["token"][b, j])] for j in range(W)]
                    for b in range(B)]
        ref_last, ref_done = ref["token"], ref["done"]
    assert hist.cpu().tolist() == ref_hist
    assert ref_done.any()


def _growth_inputs(g, B, W, depth, V, dt):
    x = [rows(g, B, 1 if d == 0 else W, V, dt) for d in range(depth)]
    return [v.cuda() for v in x], ints(g, (B, W, 33))


def _grow(growth, xs, V, stream=None):
    for x in xs:
        growth.level(x, V=V, stream=stream)
    return growth.tree(stream=stream)


def test_growth_captured_and_replayed():
    """A whole tree in one graph, states included; every replay against an eager growth."""
    note("growth graph")
    g = torch.Generator().manual_seed(59)
    B, depth, W, K, M, V = 2, 4, 3, 8, 16, 3000
    xs, st = _growth_inputs(g, B, W, depth, V, torch.bfloat16)
    growth = hs.TreeGrowth(B, depth, W, K, M, states=[st], device="cuda")
    _grow(growth, xs, V)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _grow(growth, xs, V)
    for seed in range(4):
        new, s0 = _growth_inputs(torch.Generator().manual_seed(seed), B, W, depth, V, torch.bfloat16)
        for a, b in zip(xs, new):
            a.copy_(b)
        st.copy_(s0)
        graph.replay()
        eager = hs.TreeGrowth(B, depth, W, K, M, states=[s0], device="cuda")
        want = _grow(eager, new, V)
        torch.cuda.synchronize()
        assert torch.equal(st, s0)
        assert all(torch.equal(out[k], want[k]) for k in want), seed


def test_two_growths_on_two_streams_and_a_restart():
    note("two growths")
    g = torch.Generator().manual_seed(61)
    B, depth, W, K, M = 2, 3, 4, 9, 12
    main = torch.cuda.current_stream()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = []
    for V, dt in ((5000, torch.float16), (1201, torch.float32)):
        xs, st = _growth_inputs(g, B, W, depth, V, dt)
        jobs.append((xs, st, st.clone(), V, hs.TreeGrowth(B, depth, W, K, M, states=[st], device="cuda")))
    jobs[0][4].level(jobs[1][0][0], V=1201)   # a tree that is given up, of another row length and type
    with pytest.raises(ValueError):
        jobs[0][4].tree()
    jobs[0][4].restart()
    jobs[0][1].copy_(jobs[0][2])
    for s in sides:
        s.wait_stream(main)
    outs = [None, None]
    for d in range(depth):
        for (xs, _, _, V, growth), s in zip(jobs, sides):
            growth.level(xs[d], V=V, stream=s)
    for i, ((_, _, _, _, growth), s) in enumerate(zip(jobs, sides)):
        outs[i] = growth.tree(stream=s)
        main.wait_stream(s)
    for (xs, st, s0, V, _), out in zip(jobs, outs):
        eager = hs.TreeGrowth(B, depth, W, K, M, states=[s0], device="cuda")
        want = _grow(eager, xs, V)
        assert torch.equal(st, s0)
        assert all(torch.equal(out[k], want[k]) for k in want)


def test_calls_that_make_their_tensors_for_another_stream():
    note("made for a stream")
    g = torch.Generator().manual_seed(67)
    V = 4000
    x, s = rows(g, 2, 3, V, torch.bfloat16).cuda(), scores(g, 2, 3).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [hs.beam_step(x, s, 7, V=V, stream=side) for _ in range(3)]
    with torch.cuda.stream(side):
        grown_to = [torch.stack([o[k] for o in outs]) for k in ("score", "parent", "token")]
    tree = hs.draft_tree(*grown_to, 9, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = hs.beam_step(x, s, 7, V=V)
    assert all(torch.equal(o[k], want[k]) for o in outs for k in want)
    ref = hs.draft_tree(*grown_to, 9)
    assert all(torch.equal(tree[k], ref[k]) for k in ref)


@pytest.mark.parametrize("K", [9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("mixed", [False, True])
def test_reorder_slots_shared_by_waves(K, mixed):
    """Many slots into other buffers, short rows and long, counted; with a tensor in place among them too."""
    note("shared slots K=%d mixed=%d" % (K, mixed))
    g = torch.Generator().manual_seed(K)
    W = K if mixed else 7
    src = [ints(g, (3, W, 2, T, D), torch.int16) for T, D in ((1, 8), (5, 33), (40, 64), (300, 33), (61, 100))]
    dst = [ints(g, (3, K) + tuple(s.shape[2:]), torch.int16) for s in src]
    parent = torch.randint(-1, W + 1, (3, K), generator=g, dtype=torch.int32)
    for count in (None, torch.tensor([1, 400, 37], dtype=torch.int32)):
        out = [d.clone() for d in dst]
        inp = [s.clone() for s in src]
        if mixed:
            out[2] = inp[2]
        want = []
        for s, d in zip(src, [src[2] if mixed and i == 2 else d for i, d in enumerate(dst)]):
            w = d.clone()
            for b in range(3):
                n = s.shape[3] if count is None else int(count[b])
                for j in range(K):
                    if 0 <= int(parent[b, j]) < W:
                        w[b, j, :, :n] = s[b, int(parent[b, j]), :, :n]
            want.append(w)
        hs.beam_reorder(inp, parent.cuda(), count=None if count is None else count.cuda(), axis=3, out=out)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("W", [1, 3])
@pytest.mark.parametrize("T,score", [(1e14, -1.0), (1e16, -1.0), (1e30, -1.0), (1.0, -1e16), (1.0, -1e17),
                                     (1.0, -3.4e38)])
def test_step_logits_that_score_the_same(dtype, W, T, score):
    """Temperatures and scores at which fp64 cannot tell a beam's continuations apart, and rows of many units:
    the larger logit still ranks first, wherever in the row it stands. (The beams' own scores are far enough
    apart that every slot continues the first one.)"""
    note("logits that score the same %s W=%d T=%g score=%g" % (dtype, W, T, score))
    g = torch.Generator().manual_seed(89)
    V = 151936
    x = rows(g, 1, W, V, DTYPES[dtype])
    s = torch.full((1, W), score) * torch.tensor([1.0, 1.5, 2.0])[:W] if score > -1e38 else \
        torch.tensor([[score, float("-inf"), torch.finfo(torch.float32).min]])[:, :W]
    for K in (1, 10, 64):
        got = check_step(x, s, K, V, T=T)
        assert got["parent"][0].tolist() == [0] * K


def test_step_of_more_workgroups_than_a_launch():
    """65535 queries of 64 beams that share one row of logits: 18.9 million workgroups, 2^24 a launch."""
    note("many workgroups: step")
    g = torch.Generator().manual_seed(97)
    B, W, V, K = 65535, 64, 70000, 5
    x = rows(g, 1, 1, V, torch.bfloat16)
    s = torch.stack([scores(g, 1, W)[0] for _ in range(3)])
    s[1, 1:] = float("-inf")
    out = hs.beam_step(x.cuda().expand(B, W, -1), s.cuda()[torch.arange(B, device="cuda") % 3], K, V=V)
    ref = beam.beam_step(x.expand(3, W, -1)[:, :, :V].double().numpy(), s.numpy(), K)
    torch.cuda.synchronize()
    same_step({k: v[:3].cpu().numpy() for k, v in out.items()}, ref)
    for v in out.values():
        v = v.view(B // 3, 3, K)
        assert torch.equal(v, v[:1].expand_as(v))


@pytest.mark.parametrize("K", [1, 2])
def test_reorder_of_more_workgroups_than_a_launch(K):
    note("many workgroups: reorder K=%d" % K)
    B, W, H = 65535, 2, 1030
    x = torch.arange(B * W * H * 2, dtype=torch.int32, device="cuda").to(torch.uint8).view(B, W, H, 2)
    parent = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda").expand(B, W).contiguous()[:, :K]
    count = torch.arange(B, dtype=torch.int32, device="cuda") % 3 - 1    # -1, 0 and 1 of one unit
    want = x.clone()
    want[2::3, :K, :, 0] = x[2::3].flip(1)[:, :K, :, 0]
    hs.beam_reorder(x[..., :1], parent, count=count, axis=3)
    assert torch.equal(x, want)


def test_growth_made_and_used_at_once_on_another_stream():
    """The current stream is busy when the growth is made, and its memory held NaN before: the first level, on
    a stream that waits for nothing, has the root's scores all the same."""
    note("growth on a stream of its own")
    g = torch.Generator().manual_seed(101)
    B, depth, W, K, M, V = 2, 3, 4, 8, 12, 3000
    xs, st = _growth_inputs(g, B, W, depth, V, torch.bfloat16)
    s0 = st.clone()
    side = torch.cuda.Stream()
    busy = torch.zeros(1 << 28, device="cuda")
    was = [torch.full((B, 1), float("nan"), device="cuda") for _ in range(256)]
    torch.cuda.synchronize()
    del was
    for _ in range(50):
        busy.add_(1.0)                             # 2 GB each
    growth = hs.TreeGrowth(B, depth, W, K, M, states=[st], device="cuda")
    out = _grow(growth, xs, V, stream=side)
    torch.cuda.synchronize()
    want = _grow(hs.TreeGrowth(B, depth, W, K, M, states=[s0], device="cuda"), xs, V)
    assert torch.equal(st, s0)
    assert all(torch.equal(out[k], want[k]) for k in want)


def logits_of(dtype):
    """Logits of a 16-byte vector and of a chunk of 256, and a row length of an odd number of chunks (the last slice
    is short) from which on 258 rows are cut into slices of two."""
    return (4, 1024, 39001) if dtype == "f32" else (8, 2048, 70001)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T", [1.0, 0.3])
def test_step_slices_of_two_chunks(dtype, T):
    """What one chunk of a slice holds against the other: nothing, the lowest value, logits higher by little, by
    much and by nearly the type's range, no number."""
    note("two chunks %s T=%g" % (dtype, T))
    dt = DTYPES[dtype]
    _, chunk, V = logits_of(dtype)
    g = torch.Generator().manual_seed(103)
    B, W, K = 258, 1, 6
    x = rows(g, B, W, V, dt)
    z = x[:, 0, :V]
    place = torch.arange(V) // chunk
    low, far = torch.finfo(dt).min, {"f32": 3e38, "bf16": 3e38, "f16": 6e4}[dtype]
    high = {"f32": 1e6, "bf16": 1e6, "f16": 3e4}[dtype]
    nan, inf = float("nan"), float("inf")
    for b in range(B):
        half = place % 2 == b % 2                      # the first or the second chunk of a slice
        if b // 2 % 2:
            half &= place // 2 % 3 == 1                # of some slices
        one = int(torch.randint(0, len(place) // chunk, (1,), generator=g)) // 2 * 2 + b % 2
        at = min(one * chunk + int(torch.randint(0, chunk, (1,), generator=g)), V - 1)
        kind = b // 4 % 12
        if kind == 0:
            z[b, half] = -inf
        elif kind == 1:
            z[b, half] = low
        elif kind in (2, 3, 4, 5):                     # about the 4 (in log2) at which the offset moves
            z[b, half] = (z[b, half].float() + (2.0, 3.0, 6.0, 40.0)[kind - 2]).to(dt)
        elif kind == 6:
            z[b, half] = (z[b, half].float() + high).to(dt)
        elif kind == 7:
            z[b, half] = far
        elif kind == 8:
            z[b, half] = -far
        elif kind == 9:
            z[b, at] = nan if b % 8 < 4 else inf
        elif kind == 10:                               # one logit in all
            z[b] = -inf
            z[b, at] = -3.0
        else:                                          # one above the lowest
            z[b] = low
            z[b, at] = 1.5
    check_step(x, scores(g, B, W), K, V, T=T)


def normaliser_error(z, T, dtype):
    """How far log softmax(z / T) may be off for fp64 logits z of one row, |z / T| log2(e) <= 4096: the kernel's terms
    2^x, x = z c - off, u = 2^-24, each a share p of the sum.
      - a term's exponential: 2 u (one unit in the last place); its exponent: two roundings of at most |x| u, and
        2^-35 |z c| of c's lower part, times ln 2. off lies less than 1 above and 4 below the slice's
        maximum, so |x| <= (max - z) c + 4. One term of each unit (the largest) has neither: it is replaced
        in fp64, by a series of degree 8 in |f| <= ln 2 / 2: f^9 / 9! of 2^-1/2, 2.8e-10 of itself;
      - the log2 E additions of a vector's terms in fp32: u of the sum each, and never more than the smaller addend
        (the larger one is a number the sum could be rounded to), so that a term much larger than its vector's
        others is kept;
      - the logarithm 1e-11 (in log2), and fp64 roundings: 3e-10 with the 2.8e-10 above."""
    E = 4 if dtype == "f32" else 8
    u, add = 2.0 ** -24, 2 if dtype == "f32" else 3
    c = 1.0 / (T * np.log(2.0))
    n = -(-len(z) // (E * 256)) * E * 256
    z = np.concatenate([z, np.full(n - len(z), -np.inf)])
    m = z.max()
    p = np.exp((z - m) / T)
    p /= p.sum()
    with np.errstate(invalid="ignore"):
        e = np.where(p > 0, p * (2 * u + np.log(2.0) * (2 * u * ((m - z) * c + 4) + 2.0 ** -35 * np.abs(z) * c)), 0.0)
    vec = np.arange(n) // E
    unit = vec // 256 * 4 + vec % 64 // 16
    for k in range(unit[-1] + 1):
        mine = np.flatnonzero(unit == k)
        e[mine[np.argmax(z[mine])]] = 0.0
    of = p.reshape(-1, E)
    sums = np.minimum(add * u * of.sum(1), add * (of.sum(1) - of.max(1)))
    return e.sum() + sums.sum() + 3e-10


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B", [6, 258])
def test_step_normalisers(dtype, B):
    """Scores near 0, where fp32 shows what the normalisers are good to: flat rows, a model's, and rows of one or two
    logits that have nearly all of the mass."""
    note("normalisers %s B=%d" % (dtype, B))
    dt = DTYPES[dtype]
    _, _, V = logits_of(dtype)
    g = torch.Generator().manual_seed(107 + B)
    x = rows(g, B, 1, V, dt, scale=1.0)
    T, K = 0.9, 2
    for b in range(B):
        z = torch.randn(V, generator=g)
        if b % 6 == 0:
            z *= 0.3
        elif b % 6 == 1:
            z *= 3.0
            z[torch.randint(0, V, (20,), generator=g)] += 8.0
        elif b % 6 == 2:                               # a third banned, the rest below 0
            z = torch.log_softmax(z * 2.0, 0)
            z[::3] = float("-inf")
        else:                                          # one or two logits, at any distance from an integer
            at = torch.randint(0, V, (b % 6 - 2 if b % 6 < 5 else 1,), generator=g)
            z[at] = 24.0 + 8.0 * torch.rand(1, generator=g)
            if b % 6 == 5:
                z -= 300.0
        x[b, 0, :V] = z.to(dt)
    ref = np.stack([np.sort(beam.row_log_softmax(x[b, 0, :V].double().numpy(), T))[::-1][:K] for b in range(B)])
    s = torch.from_numpy((-ref[:, :1]).astype(np.float32))
    out = hs.beam_step(x.cuda(), s.cuda(), K, V=V, temperature=T)["score"].cpu().double().numpy()
    want = s.double().numpy() + ref
    for b in range(B):
        tol = normaliser_error(x[b, 0, :V].double().numpy(), T, dtype) + 2.0 ** -24 * np.abs(want[b])
        assert np.all(np.abs(out[b] - want[b]) <= tol), (b, np.abs(out[b] - want[b]), tol)
