"""GPU parity of the calls that verify a draft, against oracle/draft.py in fp64.

Tolerances. Paths, tokens and lengths of hs_verify are exact: its weights are fp64 and good to 1.1e-12, so that of
a number's 2^53 values fewer than V 1.1e-12 lie where the two could differ."""
import numpy as np
import pytest
import torch

import paper_2510_20064_amd as hs
from oracle import draft

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def note(msg):
    print("\n[case] " + msg, flush=True)


# ---- hs_verify ------------------------------------------------------------------------------------------

def rows(g, B, M, V, dt, pad=8, scale=3.0):
    """[B][M][ld] logits, ld a multiple of 8, NaN behind V."""
    ld = (V + pad - 1) // pad * pad
    x = torch.full((B, M, ld), float("nan"), dtype=dt)
    x[:, :, :V] = (torch.randn((B, M, V), generator=g) * scale).to(dt)
    return x


def tree(g, B, M, V, z, odd=True):
    """Random parents, and tokens that mostly are their parents' likely ones; some out of range, some repeated."""
    parent = torch.full((B, M), -1, dtype=torch.int32)
    token = torch.full((B, M), -1, dtype=torch.int32)
    best = z[:, :, :V].float().nan_to_num(-9e9).topk(min(V, 8), 2).indices
    for n in range(1, M):
        up = (torch.rand(B, generator=g) ** 2 * n).long().clamp(max=n - 1)
        parent[:, n] = up.int()
        k = torch.randint(0, best.shape[2], (B,), generator=g)
        token[:, n] = best[torch.arange(B), up, k].int()
        if odd and n % 7 == 5:
            token[:, n] = torch.randint(-2, V + 2, (B,), generator=g).int()
    return parent, token


def numbers(g, B, M):
    return torch.rand((B, M), generator=g, dtype=torch.float64)


def check_verify(z, token, u, V, parent=None, drafter=None, count=None, T=1.0, mode=hs.SAMPLE, depth=None, ref=True,
                 **kw):
    up = lambda t: None if t is None else t if t.is_cuda else t.cuda()  # noqa: E731
    out = hs.verify(up(z), up(token), up(u), parent=up(parent), drafter=up(drafter), count=up(count), V=V,
                    temperature=T, mode=mode, depth=depth, **kw)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    if ref:
        num = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        want = draft.verify(z.cpu()[:, :, :V].double().numpy(), num(token), num(u), parent=num(parent),
                            drafter=None if drafter is None else drafter.cpu()[:, :, :V].double().numpy(),
                            count=num(count), T=T, greedy=mode == hs.GREEDY, depth=depth)
        for k in want:
            assert np.array_equal(got[k], want[k]), (k, got[k], want[k])
    return got


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("mode", [hs.SAMPLE, hs.GREEDY])
@pytest.mark.parametrize("B,M,V", [(1, 1, 1), (1, 2, 1), (2, 3, 7), (3, 64, 9), (2, 10, 1023), (2, 10, 2048),
                                   (2, 61, 2049), (5, 17, 4095), (2, 9, 50257)])
def test_verify_tree_sizes(dtype, mode, B, M, V):
    note("verify tree %s mode=%d B=%d M=%d V=%d" % (dtype, mode, B, M, V))
    g = torch.Generator().manual_seed(B * 1000 + M * 100 + V)
    z = rows(g, B, M, V, DTYPES[dtype])
    parent, token = tree(g, B, M, V, z)
    lengths = [check_verify(z, token, numbers(g, B, M), V, parent=parent, T=0.7, mode=mode)["length"]
               for _ in range(3)]
    assert M < 10 or mode == hs.GREEDY or max(x.max() for x in lengths) > 1


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B,M,V", [(1, 1, 5), (1, 2, 1), (2, 3, 7), (1, 64, 9), (2, 5, 1023), (4, 9, 2048),
                                   (2, 6, 2049), (7, 5, 4095), (3, 9, 50257)])
def test_verify_chain_sizes(dtype, B, M, V):
    note("verify chain %s B=%d M=%d V=%d" % (dtype, B, M, V))
    g = torch.Generator().manual_seed(B * 1000 + M * 100 + V + 1)
    z = rows(g, B, M, V, DTYPES[dtype])
    y = (z[:, :M - 1].float() + 0.5 * torch.randn(z[:, :M - 1].shape, generator=g)).to(z.dtype)
    token = torch.full((B, M), -1, dtype=torch.int32)
    if M > 1:
        q = torch.softmax(y[:, :, :V].float() / 0.8, 2)
        token[:, 1:] = torch.multinomial(q.reshape(-1, V), 1, generator=g).reshape(B, M - 1).int()
    for _ in range(3):
        u = numbers(g, B, M)
        check_verify(z, token, u, V, drafter=y if M > 1 else None, T=0.8)
        check_verify(z, token, u, V, T=0.8)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("drafted", [False, True])
def test_verify_longest_rows(dtype, drafted):
    V = (1 << 19) if dtype == "f32" else (1 << 20)
    note("verify longest rows %s drafter=%d" % (dtype, drafted))
    g = torch.Generator().manual_seed(5)
    z = rows(g, 1, 2, V, DTYPES[dtype], scale=0.5)
    y = rows(g, 1, 1, V, DTYPES[dtype], scale=0.5) if drafted else None
    for k in range(4):
        u = numbers(g, 1, 2)
        u[0, 0] = [0.0, 1.0 - 2.0 ** -53, 0.5, 0.123][k]
        check_verify(z, torch.tensor([[-1, 77777 * k]], dtype=torch.int32), u, V, drafter=y)


@pytest.mark.parametrize("T", [1e-30, 1e-3, 0.25, 1.4426950408889634, 30.0, 1e30])
def test_verify_temperatures(T):
    note("verify temperature %g" % T)
    g = torch.Generator().manual_seed(7)
    z = rows(g, 3, 9, 3001, torch.float32)
    z[:, 3, :5] = -float("inf")
    parent, token = tree(g, 3, 9, 3001, z)
    check_verify(z, token, numbers(g, 3, 9), 3001, parent=parent, T=T)
    check_verify(z, token, numbers(g, 3, 9), 3001, drafter=rows(g, 3, 8, 3001, torch.float32), T=T)


def test_verify_flat_rows_at_the_ends():
    """Every logit the same: borders at v / V exactly, where the first number above each is drawn."""
    note("verify flat rows")
    V = 8192  # a power of two: its running sums are exact
    z = torch.zeros((1, 2, V), dtype=torch.bfloat16)
    token = torch.tensor([[-1, -1]], dtype=torch.int32)
    for v in (0, 1, 2047, 2048, 4095, 8191):
        u = torch.tensor([[v / V, 0.5]], dtype=torch.float64)
        assert check_verify(z, token, u, V)["token"][0, 0] == v
        if v:
            u[0, 0] = np.nextafter(v / V, 0.0)
            assert check_verify(z, token, u, V)["token"][0, 0] == v - 1
    u = torch.tensor([[1.0 - 2.0 ** -53, 0.5]], dtype=torch.float64)
    assert check_verify(z, token, u, V)["token"][0, 0] == V - 1


@pytest.mark.parametrize("low", [-float("inf"), "min"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_verify_masks(low, dtype):
    """Masks of -inf and of the lowest value: whole slices, all but one token, all but the children's."""
    note("verify masks %s %s" % (low, dtype))
    dt, V = DTYPES[dtype], 9000
    low = torch.finfo(dt).min if low == "min" else low
    g = torch.Generator().manual_seed(11)
    z = rows(g, 4, 6, V, dt)
    z[0, :, :5000] = low
    z[0, :, 7000:V] = low
    z[1, :, :V] = low
    z[1, :, 4321] = 1.0
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2]] * 4, dtype=torch.int32)
    token = torch.randint(0, V, (4, 6), generator=g).int()
    token[1, 3:] = 4321
    z[2, :, :V] = low
    for n in range(6):  # only the children of each node
        kids = [int(t) for t, p in zip(token[2], parent[2]) if p == n]
        z[2, n, kids or [17]] = 0.5
    for _ in range(4):
        got = check_verify(z, token, numbers(g, 4, 6), V, parent=parent)
        assert got["length"][2] == 3 and got["token"][2, 2] == 17
    u = torch.full((4, 6), 1.0 - 2.0 ** -53, dtype=torch.float64)
    got = check_verify(z, token, u, V, parent=parent)
    assert got["length"][2] == 3
    y = z[:, :5].clone()
    check_verify(z, token, u, V, drafter=y)  # p = q: accepted, whatever has weight


def test_verify_rows_without_a_distribution():
    note("verify rows without a distribution")
    V = 5000
    for bad in (float("nan"), float("inf"), "none"):
        for at in (0, 77, 4999):
            for n in (0, 2):
                g = torch.Generator().manual_seed(13)
                z = rows(g, 2, 4, V, torch.float32)
                if bad == "none":
                    z[0, n, :V] = -float("inf")
                else:
                    z[0, n, at] = bad
                token = torch.tensor([[-1, 5, 77, 9]] * 2, dtype=torch.int32)
                parent = torch.tensor([[-1, 0, 0, 2]] * 2, dtype=torch.int32)
                z[:, 0, 77] += 30.0
                for mode in (hs.SAMPLE, hs.GREEDY):
                    check_verify(z, token, numbers(g, 2, 4), V, parent=parent, mode=mode)
                y = rows(g, 2, 3, V, torch.float32)
                check_verify(z, token, numbers(g, 2, 4), V, drafter=y)
                check_verify(rows(g, 2, 4, V, torch.float32), token, numbers(g, 2, 4), V, drafter=z[:, :3])


@pytest.mark.parametrize("depth", [0, 1, 2, 4])
def test_verify_depth_ends_the_draft(depth):
    """Nodes behind the depth are no part of it: their tokens may be drawn."""
    note("verify depth %d" % depth)
    g = torch.Generator().manual_seed(17)
    B, M, V = 16, 12, 40
    z = rows(g, B, M, V, torch.bfloat16)
    parent, token = tree(g, B, M, V, z, odd=False)
    token[:, 4] = token[:, 3]
    for mode in (hs.SAMPLE, hs.GREEDY):
        check_verify(z, token, numbers(g, B, M), V, parent=parent, depth=depth, mode=mode)
    y = rows(g, B, M - 1, V, torch.bfloat16)
    check_verify(z, token, numbers(g, B, M), V, drafter=y, depth=depth)


def test_verify_counts_and_strange_parents():
    note("verify counts and parents")
    g = torch.Generator().manual_seed(19)
    B, M, V = 9, 8, 300
    z = rows(g, B, M, V, torch.float16)
    parent, token = tree(g, B, M, V, z)
    count = torch.tensor([0, 1, 2, 3, 8, 100, -5, 7, 8], dtype=torch.int32)
    parent[4] = torch.tensor([3, 5, 0, 2, 99, 1, -7, 2])  # children before their parents, a loop, none
    parent[8] = torch.tensor([0, 0, 0, 0, 0, 0, 0, 0])
    z[1, 1:] = float("nan")  # not read
    for _ in range(4):
        check_verify(z, token, numbers(g, B, M), V, parent=parent, count=count, T=0.5)
        check_verify(z, token, numbers(g, B, M), V, drafter=rows(g, B, M - 1, V, torch.float16), count=count)


def test_verify_strides_and_streams():
    """Padded and broadcast views, the drafter's rows in the target's buffer, another stream, calls in a row."""
    note("verify strides and streams")
    g = torch.Generator().manual_seed(23)
    B, M, V = 3, 5, 1000
    big = rows(g, B, 2 * M, V + 24, torch.bfloat16).cuda()
    z, y = big[:, ::2], big[:, 1:2 * M - 2:2]
    token = torch.randint(0, V, (B, M), generator=g).int()
    u = numbers(g, B, M)
    check_verify(z, token, u, V, drafter=y)
    check_verify(z[:1].expand(B, M, z.shape[2]), token, u, V)
    check_verify(z[:, :1].expand(B, M, z.shape[2]), token, u, V, drafter=y[:, :1].expand(B, M - 1, y.shape[2]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_verify(z, token.cuda(), u.cuda(), V, drafter=y, stream=s)
    with torch.cuda.stream(s):
        check_verify(z, token, u, V, drafter=y)


@pytest.mark.parametrize("drafted", [False, True])
def test_verify_captured(drafted):
    """A captured call, replayed on other inputs with eager calls between."""
    note("verify captured drafter=%d" % drafted)
    g = torch.Generator().manual_seed(29)
    B, M, V = 4, 6, 3000
    z = rows(g, B, M, V, torch.bfloat16).cuda()
    y = rows(g, B, M - 1, V, torch.bfloat16).cuda() if drafted else None
    token, u = torch.zeros((B, M), dtype=torch.int32, device="cuda"), numbers(g, B, M).cuda()
    plan = hs.Verify(z, token, u, drafter=y, V=V)
    plan.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    for k in range(4):
        token.copy_(z.argmax(2).roll(1, 1).int() if k % 2 else torch.randint(0, V, (B, M), generator=g).int())
        u.copy_(numbers(g, B, M))
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.cpu().numpy() for n, t in plan.out.items()}
        want = check_verify(z, token, u, V, drafter=y)
        for n in want:
            assert np.array_equal(got[n], want[n]), (k, n)


def test_verify_far_rows():
    """Offsets beyond 32 bits: a view whose queries lie 3 GB apart."""
    note("verify far rows")
    g = torch.Generator().manual_seed(31)
    V, B, M = 2000, 3, 3
    apart = 3 * (1 << 29)
    buf = torch.empty(2 * apart + 4 * 2048, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(buf, (B, M, 2000), (apart, 2048, 1))
    z.copy_(rows(g, B, M, V, torch.bfloat16))
    token = torch.randint(0, V, (B, M), generator=g).int()
    check_verify(z, token, numbers(g, B, M), V)


def test_verify_most_queries():
    note("verify most queries")
    g = torch.Generator().manual_seed(37)
    B, M, V = 65535, 2, 8
    z = rows(g, B, M, V, torch.bfloat16)
    token = torch.randint(0, V, (B, M), generator=g).int()
    u = numbers(g, B, M)
    got = check_verify(z, token, u, V, ref=False)
    some = torch.randint(0, B, (200,), generator=g)
    want = draft.verify(z[some, :, :V].double().numpy(), token[some].numpy(), u[some].numpy())
    for k in want:
        assert np.array_equal(got[k][some.numpy()], want[k]), k
