"""GPU parity of the calls that verify a draft, against oracle/draft.py in fp64.

Tolerances. Paths, tokens and lengths of hs_verify are exact: its weights are fp64 and good to 1.1e-12, so that of
a number's 2^53 values fewer than V 1.1e-12 lie where the two could differ. Codes and scales of hs_cache_append are
exact. An output of hs_tree_attention over n tokens, o = sum p v, may be off by
  eps / 2 |o|, its rounding (bf16 2^-8, fp16 2^-11; below the type's least normal number, where steps are as wide as just
  above it, eps / 2 of that: fp16 2^-25, so that -2.94e-6, between steps of 2^-24, is held as -2.92e-6), and of sum p |v|
    2^-11, a weight's rounding to fp16 (what is below 2^-36 of the largest, n 2^-37 at most, is in the sums' share),
    2 (dim + 8) 2^-24 a, the scores' fp32 sums of products, a = the largest scale * sum |q| |k|, in weight and sum,
    2 (2^-22 + 2^-23 + 4 * 2^-24 a), exponential, scale and the three roundings on the way to it, and
    2 (n + 300) 2^-24, the fp32 sums over n tokens and 128 splits of a row."""
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


def shallow(parent, depth):
    """The parents of a tree whose nodes further than `depth` from the root hang from it instead, and their depths."""
    far = torch.zeros(parent.shape, dtype=torch.long)
    parent = parent.clone()
    rows = torch.arange(parent.shape[0])
    for n in range(1, parent.shape[1]):
        deep = far[rows, parent[:, n].long()] >= depth
        parent[deep, n] = 0
        far[:, n] = far[rows, parent[:, n].long()] + 1
    return parent


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("mode", [hs.SAMPLE, hs.GREEDY])
def test_verify_large_trees(dtype, mode):
    """Calls so large that only the rows on the paths are read, with ragged and empty drafts, rows without a
    distribution and nodes behind the depth."""
    note("verify large trees %s mode=%d" % (dtype, mode))
    g = torch.Generator().manual_seed(43)
    B, M, V, depth = 32, 48, 40013, 3
    z = rows(g, B, M, V, DTYPES[dtype])
    parent, token = tree(g, B, M, V, z)
    parent = shallow(parent, depth)
    count = torch.randint(1, M + 1, (B,), generator=g).int()
    count[5], count[6], count[7] = 0, 1, M
    z[3, 1:4, 17] = float("nan")
    z[4, 0, :V] = -float("inf")
    for k in range(3):
        got = check_verify(z, token, numbers(g, B, M), V, parent=parent, count=count if k else None, mode=mode, T=0.6,
                           depth=depth)
        check_verify(z, token, numbers(g, B, M), V, parent=parent, count=count, mode=mode, depth=1)
    assert mode == hs.GREEDY or got["length"].max() > 1
    # each node's first child has its likeliest token: longer paths
    first = torch.full((B, M), M, dtype=torch.long).scatter_reduce(1, parent[:, 1:].long(), torch.arange(1, M).expand(B, -1),
                                                                   "amin")
    best = z[:, :, :V].float().nan_to_num(-9e9).argmax(2)
    for b in range(B):
        for n in range(M):
            if first[b, n] < M:
                token[b, first[b, n]] = best[b, n]
    got = check_verify(z, token, numbers(g, B, M), V, parent=parent, mode=mode, T=0.2, depth=depth)
    assert got["length"].max() == depth + 1


@pytest.mark.parametrize("mode", [hs.SAMPLE, hs.GREEDY])
def test_verify_large_trees_of_long_rows(mode):
    """Rows of more slices than a wave holds two a lane."""
    note("verify large trees of long rows mode=%d" % mode)
    g = torch.Generator().manual_seed(53)
    B, M, V, depth = 6, 40, 300007, 2
    z = rows(g, B, M, V, torch.bfloat16)
    parent, token = tree(g, B, M, V, z)
    parent = shallow(parent, depth)
    for count in (None, torch.tensor([40, 0, 1, 2, 39, 17], dtype=torch.int32)):
        check_verify(z, token, numbers(g, B, M), V, parent=parent, count=count, mode=mode, T=0.5, depth=depth)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("drafted", [False, True])
def test_verify_large_chains(dtype, drafted):
    note("verify large chains %s drafter=%d" % (dtype, drafted))
    g = torch.Generator().manual_seed(47)
    B, M, V = 96, 6, 70001
    z = rows(g, B, M, V, DTYPES[dtype], scale=2.0).cuda()
    y = (z[:, :M - 1].float() + 0.4 * torch.randn(z[:, :M - 1].shape, device="cuda")).to(z.dtype)
    y[:, :, V:] = float("nan")
    pick = -(-torch.rand((B, M - 1, V), device="cuda").clamp(min=1e-30).log()).log()
    token = torch.full((B, M), -1, dtype=torch.int32)
    token[:, 1:] = (y[:, :, :V].float() + pick).argmax(2).cpu().int()
    count = torch.randint(0, M + 1, (B,), generator=g).int()
    z[7, 2, 5], y[8, 1, 9] = float("nan"), float("inf")
    for k in range(2):
        got = check_verify(z, token, numbers(g, B, M), V, drafter=y if drafted else None, count=count if k else None)
        assert not drafted or got["length"].max() > 3


def test_verify_of_roots_alone_takes_a_drafter_without_rows():
    """M = 1 as a loop over drafts of any length has it: a drafter of no rows, when the plan is made and later."""
    note("verify roots with a drafter of no rows")
    g = torch.Generator().manual_seed(59)
    z, none = rows(g, 3, 1, 64, torch.float32).cuda(), torch.empty((3, 0, 64), device="cuda")
    token, u = torch.full((3, 1), -1, dtype=torch.int32, device="cuda"), numbers(g, 3, 1).cuda()
    plan = hs.Verify(z, token, u, drafter=none)
    first = {n: t.clone() for n, t in plan.run().items()}
    other = rows(g, 3, 1, 64, torch.float32).cuda()
    for drafter in (none, None):
        plan.set_logits(other, drafter)
        got, want = plan.run(), hs.verify(other, token, u)
        assert all(torch.equal(got[n], want[n]) for n in want)
        plan.set_logits(z, drafter)
        assert all(torch.equal(plan.run()[n], first[n]) for n in first)


# ---- hs_tree_attention -----------------------------------------------------------------------------------

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Draft:
    """Inputs of an attention: a pool whose unused codes are NaN, and drafts over it."""

    def __init__(self, seed, B, M, heads, kv, dim, page, lengths, dtype, tree_=True, counts=None, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.B, self.M, self.kv, self.dim, self.page = B, M, kv, dim, page
        slots = max(1, -(-max(lengths) // page))
        pages = B * slots + spare
        x = (torch.randn((pages, kv, page, dim), generator=g) * 80).clamp(-448, 448).to(torch.float8_e4m3fn)
        y = (torch.randn((pages, kv, dim, page), generator=g) * 80).clamp(-448, 448).to(torch.float8_e4m3fn)
        self.ck, self.cv = x.view(torch.uint8), y.view(torch.uint8)
        self.sk = torch.exp2(torch.randint(-8, -4, (pages, kv), generator=g).float())
        self.sv = torch.exp2(torch.randint(-9, -4, (pages, kv), generator=g).float())
        self.table = torch.randperm(pages, generator=g)[:B * slots].reshape(B, slots).int()
        self.length = torch.tensor(lengths, dtype=torch.int32)
        used = torch.zeros((pages, page), dtype=torch.bool)
        for b, n in enumerate(lengths):
            for j in range(slots):
                used[self.table[b, j].long(), :max(0, min(page, n - j * page))] = True
        self.ck[~used[:, None].expand(pages, kv, page)] = 0x7F
        self.cv.copy_(torch.where(used[:, None, None], self.cv, torch.tensor(0xFF, dtype=torch.uint8)))
        qkv = torch.randn((B, M, heads + 2 * kv, dim), generator=g).to(dtype)
        self.q, self.k, self.v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:]
        self.mask = None
        if tree_:
            self.mask = torch.zeros((B, M), dtype=torch.int64)
            for n in range(M):
                up = (torch.rand(B, generator=g) * n).long()
                bits = self.mask[torch.arange(B), up] if n else torch.zeros(B, dtype=torch.int64)
                self.mask[:, n] = bits | (1 << n if n < 63 else -(1 << 63))
        self.count = None if counts is None else torch.tensor(counts, dtype=torch.int32)
        self.scale = 1.5 * dim ** -0.5

    def gpu(self):
        up = lambda t: None if t is None else t if t.is_cuda else t.cuda()  # noqa: E731
        cache = hs.PagedCache(*[up(t) for t in (self.ck, self.cv, self.sk, self.sv)])
        out = torch.full(self.q.shape, -77.0, dtype=self.q.dtype, device="cuda")
        return dict(q=up(self.q), k=up(self.k), v=up(self.v), cache=cache, table=up(self.table), length=up(self.length),
                    mask=up(self.mask), count=up(self.count), scale=self.scale, out=out)

    def check(self, got=None, **kw):
        if got is None:
            got = hs.tree_attention(**dict(self.gpu(), **kw))
            torch.cuda.synchronize()
        num = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
        ref, mean, most = draft.attention(f64(self.q), f64(self.k), f64(self.v), num(self.ck), num(self.cv),
                                          num(self.sk), num(self.sv), num(self.table), num(self.length),
                                          mask=num(self.mask), count=num(self.count), scale=self.scale)
        y = got.cpu().double().numpy()
        for b in range(self.B):
            n = self.M if self.count is None else min(max(int(self.count[b]), 0), self.M)
            assert np.all(y[b, n:] == -77.0), b  # left as they were
            o, r = y[b, :n], ref[b, :n]
            bad = ~np.isfinite(r)
            assert np.array_equal(np.isnan(o), np.isnan(r)) and np.array_equal(o[bad & ~np.isnan(r)], r[bad & ~np.isnan(r)])
            a, tokens = most[b, :n][..., None], int(self.length[b]) + self.M
            rel = 2.0 ** -11 + 2 * (self.dim + 8) * 2.0 ** -24 * a + 2 * (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -22 * a) + \
                2 * (tokens + 300) * 2.0 ** -24
            tol = HALF[self.q.dtype] * np.maximum(np.abs(r), torch.finfo(self.q.dtype).tiny) + rel * mean[b, :n]
            with np.errstate(invalid="ignore"):
                over = np.where(bad, 0.0, np.abs(o - r) - tol)
            assert n == 0 or over.max() <= 0, (b, over.max(), np.unravel_index(over.argmax(), over.shape))
        return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,heads,kv,dim,page,lengths", [
    (1, 1, 1, 32, 32, [0]), (1, 1, 1, 32, 32, [1]), (1, 4, 4, 64, 32, [31, 32, 33]), (1, 8, 2, 128, 64, [63, 64, 65, 0]),
    (2, 15, 3, 64, 32, [1999, 77, 0, 511]), (3, 5, 1, 96, 128, [127, 128, 129, 300]), (7, 8, 8, 128, 256, [255, 257, 999]),
    (33, 2, 1, 160, 64, [700, 3]), (61, 4, 1, 128, 64, [1500, 64, 0]), (64, 8, 1, 64, 32, [255, 256, 257, 258]),
    (16, 3, 3, 192, 64, [513, 40]), (5, 14, 2, 224, 32, [300, 1]), (9, 16, 2, 256, 128, [777, 1000, 4]),
    (64, 2, 2, 256, 32, [95, 33]), (1, 32, 8, 128, 64, [4097])])
def test_attention_sizes(dtype, M, heads, kv, dim, page, lengths):
    note("attention %s M=%d heads=%d/%d dim=%d page=%d %s" % (dtype, M, heads, kv, dim, page, lengths))
    Draft(M * 100 + heads + dim, len(lengths), M, heads, kv, dim, page, lengths, dtype).check()
    Draft(M * 100 + heads + dim + 1, len(lengths), M, heads, kv, dim, page, lengths, dtype, tree_=False).check()


@pytest.mark.parametrize("M,heads,kv,dim,page,B,most", [
    (1, 8, 8, 64, 32, 100, 1100), (1, 8, 8, 64, 32, 100, 500), (1, 2, 2, 32, 32, 300, 2000), (2, 16, 16, 32, 32, 200, 300),
    (5, 20, 4, 64, 32, 70, 1100), (20, 8, 8, 64, 64, 66, 1300)])
def test_attention_many_queries(M, heads, kv, dim, page, B, most):
    """More queries than lanes, with lengths that differ widely, some of them zero."""
    note("attention many M=%d heads=%d/%d dim=%d B=%d most=%d" % (M, heads, kv, dim, B, most))
    g = torch.Generator().manual_seed(B + M)
    lengths = [int(n) for n in (torch.rand(B, generator=g) ** 3 * most).long()]
    lengths[0], lengths[B // 2], lengths[B - 1] = 0, most, 0
    counts = [int(n) for n in torch.randint(0, M + 1, (B,), generator=g)]
    Draft(B, B, M, heads, kv, dim, page, lengths, torch.bfloat16).check()
    Draft(B, B, M, heads, kv, dim, page, lengths, torch.float16, counts=counts).check()


@pytest.mark.parametrize("M,heads,kv,dim,page,lengths", [
    (4, 4, 1, 64, 32, [700, 5]), (17, 1, 1, 64, 32, [700, 5]), (16, 2, 1, 128, 32, [300, 1]), (11, 3, 1, 128, 64, [300, 64]),
    (64, 1, 1, 128, 32, [400]), (13, 5, 1, 128, 32, [400, 0]), (64, 2, 1, 128, 64, [600]), (43, 3, 1, 128, 64, [600]),
    (64, 4, 1, 128, 64, [600]), (52, 5, 1, 128, 64, [600, 9]), (64, 8, 1, 192, 64, [333, 64]), (64, 16, 2, 256, 32, [77]),
    (33, 4, 1, 160, 32, [500]), (64, 5, 1, 224, 64, [333, 64]), (41, 3, 1, 256, 64, [333, 64]), (16, 4, 1, 256, 32, [90])])
@pytest.mark.parametrize("slots", [0, 40])
def test_attention_row_counts(M, heads, kv, dim, page, lengths, slots):
    """Rows of a head on both sides of each variant's size, with tables for short and for long caches."""
    note("attention rows M=%d heads=%d/%d dim=%d slots=%d" % (M, heads, kv, dim, slots))
    d = Draft(M + heads, len(lengths), M, heads, kv, dim, page, lengths, torch.bfloat16)
    if slots:
        wide = torch.full((len(lengths), max(slots, d.table.shape[1])), -1, dtype=torch.int32)
        wide[:, :d.table.shape[1]] = d.table
        d.table = wide
    d.check()


@pytest.mark.parametrize("M", [1, 30])
@pytest.mark.parametrize("tokens", [127, 128, 129, 255, 256, 257, 384, 1023, 1025])
def test_attention_short_and_long_tables(M, tokens):
    note("attention tables of %d tokens M=%d" % (tokens, M))
    d = Draft(tokens + M, 2, M, 4, 2, 64, 32, [tokens, tokens // 2], torch.float16)
    d.check()


def test_attention_counts():
    note("attention counts")
    for M, counts in ((5, [0, 1, 5, 9, -3, 4]), (40, [40, 33, 32, 31, 1, 0])):
        d = Draft(M, 6, M, 6, 2, 64, 32, [100, 0, 64, 5, 33, 0], torch.bfloat16, counts=counts)
        for b, n in enumerate(counts):  # nodes behind the count hold anything
            d.k[b, max(n, 0):] = float("nan")
            d.v[b, max(n, 0):] = float("inf")
            d.mask[b, max(n, 0):] = 0
        d.check()


def test_attention_rows_that_see_nothing():
    note("attention empty rows")
    d = Draft(3, 3, 6, 4, 2, 64, 32, [0, 0, 40], torch.float16)
    d.mask[:, 1:4] = 0
    got = d.check()
    assert torch.all(got[:2, 1:4] == 0)


def test_attention_masked_nodes_may_hold_anything():
    note("attention NaN and infinities in masked nodes")
    for dtype in (torch.bfloat16, torch.float16):
        for bad in (float("nan"), float("inf"), -float("inf")):
            d = Draft(5, 2, 40, 4, 2, 64, 32, [50, 0], dtype)
            d.v[0, 7, 1, 33] = bad   # reaches those that see nodes 7 and 35
            d.v[1, 35, 0, :] = bad
            d.check()
            d = Draft(5, 2, 40, 4, 2, 64, 32, [50, 0], dtype)
            seen = torch.tensor([[(int(m) >> 9) & 1 for m in d.mask[b]] for b in range(2)]).bool()
            d.k[:, 9] = bad
            d.v[:, 9] = bad
            got = hs.tree_attention(**d.gpu()).cpu()
            assert torch.isfinite(got[~seen]).all() and not torch.isfinite(got[seen]).any()


def test_attention_large_values_of_bf16_nodes():
    """bf16's range: the nodes' values are not held in fp16."""
    note("attention large node values")
    d = Draft(7, 2, 20, 4, 2, 64, 32, [50, 0], torch.bfloat16)
    d.v *= 1e20
    d.check()
    d.v *= 1e-37
    d.check()


def test_attention_scales():
    """Pages whose scales lie far apart, scales that are no powers of two, zeros, and cached NaN."""
    note("attention scales")
    g = torch.Generator().manual_seed(8)
    d = Draft(9, 2, 3, 4, 2, 128, 32, [320, 200], torch.bfloat16)
    d.sv.copy_(torch.exp2(torch.randint(-20, 20, d.sv.shape, generator=g).float()))
    d.check()
    d.sv.copy_(torch.exp2(torch.randint(-40, 41, d.sv.shape, generator=g).float()))
    d.check()
    d.sv.copy_(torch.rand(d.sv.shape, generator=g) + 0.01)
    d.sk.copy_((torch.rand(d.sk.shape, generator=g) - 0.5) * 0.02)
    d.check()
    d.sk[d.table[0, 1].long()] = 0.0
    d.sv[d.table[0, 2].long()] = 0.0
    d.check()
    d.cv[d.table[0, 3].long(), 1, 17, 5] = 0x7F
    d.check()
    d.ck[d.table[1, 3].long(), 0, 5, 3] = 0xFF
    d.check()


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_values_of_pages_far_finer_than_others(dtype, M, heads):
    """A page whose scale is far above the others', and which has no code in half of the dimensions: there the others'
    values are all, as good as without it."""
    note("attention pages far finer %s M=%d heads=%d" % (dtype, M, heads))
    for spread in (6, 20, 27, 34, 40, 60, 79):
        d = Draft(M + spread, 3, M, heads, 1, 64, 32, [400, 33, 150], dtype)
        top = 40.0 if dtype == torch.bfloat16 else 10.0
        d.sv[:] = 2.0 ** max(top - spread, -40.0)
        d.v *= 2.0 ** (max(top - spread, -40.0) + 6)
        for p in (d.table[0, 3], d.table[0, 9], d.table[1, 0]):
            d.sv[p.long()] = 2.0 ** top
            d.cv[p.long(), 0, 32:] = torch.where((d.cv[p.long(), 0, 32:] & 0x7F) == 0x7F, d.cv[p.long(), 0, 32:], 0)
        if dtype == torch.float16:  # codes of 0 and 2: 448 * 2^10 would be no fp16
            d.cv[:, :, :32] = torch.where((d.cv[:, :, :32] & 0x7F) == 0x7F, d.cv[:, :, :32], d.cv[:, :, :32] & 0xC0)
        d.check()


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
def test_attention_any_finite_value_of_bf16_nodes(M, heads):
    """Nodes' values up to the largest bf16; and one of them alone, beside dimensions that hold cached values only."""
    note("attention huge node values M=%d heads=%d" % (M, heads))
    for e in (80, 89, 90, 100, 112, 120, 127):
        d = Draft(M + e, 3, M, heads, 1, 64, 32, [400, 33, 0], torch.bfloat16)
        d.v.copy_((d.v * 2.0 ** (e - 2)).clamp_(-3.38e38, 3.38e38))
        d.check()
    for e in (80, 92, 104):
        d = Draft(M + e, 3, M, heads, 1, 64, 32, [400, 33, 0], torch.bfloat16)
        d.v.zero_()
        d.v[:, M // 2, :, 7] = 2.0 ** e
        d.check()


class Sharp(Draft):
    """Scores that lie far apart, where a dimension may hold nothing but values of tokens of little weight. A weight is held as
    2^12 w in fp16, w relative to a maximum that is at most 2^4 (what scales differ by here) above the row's largest weight of
    any page: below 2^-14 fp16's steps are 2^-24, so that w is off by 2^-25 2^-12 = 2^-37 of that maximum, 2^-33 of the largest
    weight, and that is at most 1. Each of n tokens may so add 2^-33 |v| to an output."""

    def check(self, got=None, **kw):
        if got is None:
            got = hs.tree_attention(**dict(self.gpu(), **kw))
            torch.cuda.synchronize()
        f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
        ref, mean, most = draft.attention(f64(self.q), f64(self.k), f64(self.v), self.ck.numpy(), self.cv.numpy(),
                                          self.sk.numpy(), self.sv.numpy(), self.table.numpy(), self.length.numpy(),
                                          mask=self.mask.numpy(), scale=self.scale)
        y = got.cpu().double().numpy()
        large = max(448 * float(self.sv.abs().max()), float(self.v.abs().max()))
        for b in range(self.B):
            a, n = most[b][..., None], int(self.length[b]) + self.M
            rel = 2.0 ** -11 + 2 * (self.dim + 8) * 2.0 ** -24 * a + 2 * (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -22 * a) + \
                2 * (n + 300) * 2.0 ** -24
            tol = HALF[self.q.dtype] * np.abs(ref[b]) + rel * mean[b] + n * 2.0 ** -33 * large
            assert np.all(np.abs(y[b] - ref[b]) <= tol), (b, (np.abs(y[b] - ref[b]) - tol).max())


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
def test_attention_any_finite_key_scales(M, heads):
    """Scales of 0, smallest and largest ones, of either sign, with queries that make products large or nothing of them."""
    note("attention any key scales M=%d heads=%d" % (M, heads))
    # (the scale of the call, of the keys, what the queries are multiplied with)
    for scale, sk, size in ((0.0, None, 1e30), (0.0, -1.0, 1e30), (-0.0, None, 1.0), (1e-38, 1e-3, 1e30), (-1e-38, 1.0, 1e30),
                            (1.0, -1e-33, 1e30), (-1.0, 1e-40, 1e30), (1e-3, 0.0, 1.0), (1e-30, 1e-30, 1e30), (1.0, 1e30, 1e-31),
                            (1e-20, 1e30, 1e-12), (-1e20, 1e-30, 1e9)):
        d = Sharp(M + 5, 3, M, heads, 1, 64, 32, [400, 33, 150], torch.bfloat16)
        d.scale = scale
        d.q.copy_((d.q.float() * size).to(d.q.dtype))
        d.k.zero_()  # (the nodes' own products would not be finite)
        if sk is not None:
            d.sk[:] = sk
        d.check()
    d = Sharp(M + 5, 3, M, heads, 1, 64, 32, [400, 33, 150], torch.bfloat16)
    d.scale = 10.0
    far = d.table[0, 2:5].long()
    d.sk[far] = 3e38  # 10 times that is infinite, and codes of 0 make nothing of it
    d.ck[far] = 0
    d.check()


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
def test_attention_lowest_scores(M, heads):
    """Of tokens whose scores are all far below 0 the largest has the weight, down to the lowest fp32 (2.36e38 times log2 e)."""
    note("attention lowest scores M=%d heads=%d" % (M, heads))
    dim, page = 64, 32
    for scale in (-1e30, -1e38, -1.5e38, -2.3e38):
        code = torch.full((4, 1, page, dim), 0x38, dtype=torch.uint8)
        code[:, :, 1::2] = 0x3C  # keys of 1 and 1.5: scores of 2/3 scale and scale; the nodes' are 3/4 scale
        code[2, 0, 16] = 0x30    # one of 1/3, or of a node 1/4
        values = torch.randint(0x30, 0x40, (4, 1, dim, page), generator=torch.Generator().manual_seed(3)).to(torch.uint8)
        one = torch.ones((4, 1), device="cuda")
        cache = hs.PagedCache(code.cuda(), values.cuda(), one, one.clone())
        table = torch.tensor([[0, 1, 2, 3], [0, 1, 3, 3], [3, 3, 3, 3]], dtype=torch.int32, device="cuda")
        length = torch.tensor([128, 1, 0], dtype=torch.int32, device="cuda")
        q = torch.full((3, M, heads, dim), 1.0 / 96, dtype=torch.float32).to(torch.bfloat16).cuda()
        k = torch.full((3, M, 1, dim), 1.125, dtype=torch.bfloat16, device="cuda")
        v = torch.randn((3, M, 1, dim), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
        own = torch.tensor([[1 << n for n in range(M)]], dtype=torch.int64).expand(3, M).contiguous().cuda()
        got = hs.tree_attention(q, k, v, cache, table, length, mask=own, scale=scale)
        want = v.expand(3, M, heads, dim).clone()
        want[0] = values[2, 0, :, 16].view(torch.float8_e4m3fn).to(torch.bfloat16).cuda()  # the one of 1/3
        want[1] = values[0, 0, :, 0].view(torch.float8_e4m3fn).to(torch.bfloat16).cuda()   # 2/3, before the node's 3/4
        assert torch.equal(got, want), scale


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
@pytest.mark.parametrize("apart", [0, 2, 40])
def test_attention_large_scores(M, heads, apart):
    """Scores that fp32 holds in steps of 1/8 to 1e31: the largest token has all the weight, of early and late pages, with
    values of any scale."""
    note("attention large scores M=%d heads=%d scales 2^%d apart" % (M, heads, apart))
    dim, page, n = 64, 32, 300
    g = torch.Generator().manual_seed(17)
    for scale in (1e5, 3e7, 1e9, 1e15, 1e30, 3e36, -1e5, -1e8, -1e12, -3e36):
        code = torch.randint(0x28, 0x38, (10, 1, page, dim), generator=g).to(torch.uint8)  # 1/4 to 15/16
        values = torch.randint(0x30, 0x40, (10, 1, dim, page), generator=g).to(torch.uint8)
        best = [5, 70, 130, 299]  # of each query
        code = code.repeat(4, 1, 1, 1)
        values = values.repeat(4, 1, 1, 1)
        for b, t in enumerate(best):
            code[10 * b + t // page, 0, t % page] = 0x40 if scale > 0 else 0x10  # 2, or 1/16
        sv = torch.exp2(torch.randint(-apart, apart + 1, (40, 1), generator=g).float())
        cache = hs.PagedCache(code.cuda(), values.cuda(), torch.ones((40, 1), device="cuda"), sv.cuda())
        table = torch.arange(40).reshape(4, 10).int().cuda()
        length = torch.full((4,), n, dtype=torch.int32, device="cuda")
        q = torch.full((4, M, heads, dim), 1.0 / 64, dtype=torch.bfloat16, device="cuda")
        k = torch.full((4, M, 1, dim), 0.5, dtype=torch.bfloat16, device="cuda")
        v = torch.randn((4, M, 1, dim), generator=g).to(torch.bfloat16).cuda()
        got = hs.tree_attention(q, k, v, cache, table, length, scale=scale).cpu()
        for b, t in enumerate(best):
            p = 10 * b + t // page
            want = values[p, 0, :, t % page].view(torch.float8_e4m3fn).float() * sv[p]
            assert torch.all((got[b].float() - want).abs() <= want.abs() * 2.0 ** -7), (scale, b)


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
def test_attention_value_scales_of_zero(M, heads):
    """Values of a page whose scale is 0 are 0, and their weights count."""
    note("attention value scales of zero M=%d heads=%d" % (M, heads))
    for zero in (0.0, -0.0):
        d = Draft(M + 7, 3, M, heads, 1, 64, 32, [400, 33, 150], torch.bfloat16)
        d.sv[d.table[0, 1:9].long()] = zero
        d.sv[d.table[1].long()] = zero
        d.check()
        d.cv[d.table[0, 3].long(), 0, 20, 9] = 0x7F
        d.cv[d.table[1, 0].long(), 0, 7, 31] = 0xFF
        d.check()
        d = Draft(M + 8, 3, M, heads, 1, 64, 32, [400, 33, 150], torch.bfloat16)
        d.sv[:] = zero
        d.v.zero_()
        assert torch.all(d.check() == 0)
        d.v.fill_(1e-30)
        d.check()


@pytest.mark.parametrize("M,heads", [(1, 4), (5, 3), (20, 2), (40, 6), (61, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_small_and_large_values(dtype, M, heads):
    """Values of cache and nodes alike, from far below 1 to far above."""
    note("attention small and large values %s M=%d heads=%d" % (dtype, M, heads))
    g = torch.Generator().manual_seed(61)
    for size in (-40, -34, -27, -20, -14, -3, 5, 12) + ((25, 39) if dtype == torch.bfloat16 else ()):
        d = Draft(M + 99 + size, 3, M, heads, 1, 64, 32, [400, 33, 150], dtype)
        d.sv[:] = 2.0 ** (torch.randint(0, 2, d.sv.shape, generator=g).float() + size)
        d.v *= 2.0 ** (size + 6)
        if dtype == torch.float16 and size > 5:
            d.v.clamp_(-6e4, 6e4)
            d.cv.copy_(torch.where((d.cv & 0x7F) == 0x7F, d.cv, d.cv & 0xBF))  # codes below 2, values below 2^14
        d.check()


def test_attention_sharp_and_flat():
    """Scores from equal to far apart: one token has all the weight, and late maxima."""
    note("attention sharp and flat")
    for scale in (0.0, 1e-3, 1.0, 8.0, -2.0):
        d = Draft(10, 2, 4, 8, 2, 64, 64, [1500, 333], torch.float16)
        d.scale = scale
        d.check()


def test_attention_tables():
    """Pages that queries share, pages that are not there, lengths beyond the table and negative ones."""
    note("attention tables")
    d = Draft(11, 4, 5, 4, 2, 64, 32, [160, 160, 150, 90], torch.bfloat16)
    d.table[1, :3] = d.table[0, :3]
    d.table[1, 3] = d.table[1, 2]
    d.table[2, 1], d.table[2, 4] = -1, 99999
    d.table[3] = -7
    d.check()
    d.length[0], d.length[1] = 1 << 30, -5
    d.check()
    wide = torch.full((4, 9), -1, dtype=torch.int32)
    wide[:, :5] = d.table
    d.table = wide[:, :5]
    full = wide.cuda()
    d.check(table=full[:, :5])


@pytest.mark.parametrize("M,heads", [(1, 4), (16, 1), (5, 3), (20, 2), (30, 4), (40, 6), (61, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_scales_of_pages_that_no_query_has(dtype, M, heads):
    """Pages without a token of any query, the first of the pool among them, hold any scale: for caches that end inside a
    stage and pages that are not there, in each variant of rows."""
    note("attention scales of unused pages %s M=%d heads=%d" % (dtype, M, heads))
    for bad in (float("nan"), float("inf"), -float("inf")):
        lengths = [1, 33, 129, 0, 300, 511, 96]
        d = Draft(M + heads, len(lengths), M, heads, 1, 64, 32, lengths, dtype)
        other = [int(p) for p in range(len(d.ck)) if p not in d.table.flatten().tolist()][0]
        for t in (d.ck, d.cv, d.sk, d.sv):  # the first page is in no table
            t[[0, other]] = t[[other, 0]]
        d.table[d.table == 0] = other
        d.table[4, 2], d.table[5, 7] = -1, len(d.ck) + 3
        held = torch.zeros(len(d.ck), dtype=torch.bool)
        for b, n in enumerate(lengths):
            for p in d.table[b, :-(-n // 32)].tolist():
                if 0 <= p < len(held):
                    held[p] = True
        assert not held[0]
        d.sk[~held] = bad
        d.sv[~held] = bad
        d.check()


def test_attention_strides_and_streams():
    note("attention strides and streams")
    d = Draft(12, 3, 6, 8, 2, 128, 64, [200, 77, 0], torch.bfloat16)
    args = d.gpu()
    # heads before nodes, in and out, and the batch broadcast
    args["q"] = args["q"].transpose(1, 2).contiguous().transpose(1, 2)
    args["out"] = torch.full((3, 8, 6, 160), -77.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)[..., :128]
    d.check(got=hs.tree_attention(**args))
    d.k, d.v = d.k[:1].expand(d.k.shape), d.v[:1].expand(d.v.shape)
    d.check(k=d.k[:1].cuda().expand(d.k.shape), v=d.v[:1].cuda().expand(d.v.shape))
    s = torch.cuda.Stream()
    args = d.gpu()
    s.wait_stream(torch.cuda.current_stream())
    got = hs.tree_attention(stream=s, **args)
    s.synchronize()
    d.check(got=got)


@pytest.mark.parametrize("M", [1, 21])
def test_attention_captured(M):
    """A captured call, replayed as the cache grows, with eager calls between; two plans share a workspace in order."""
    note("attention captured M=%d" % M)
    d = Draft(13, 2, M, 8, 2, 128, 64, [4000, 3000], torch.bfloat16)
    args = d.gpu()
    plan = hs.TreeAttention(**args)
    plan.run()
    other = hs.TreeAttention(**dict(args, out=torch.empty_like(args["out"]), workspace=plan.workspace))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
        other.run()
    for n in ((1, 0), (300, 4000), (4000, 2500), (33, 64)):
        d.length = torch.tensor(n, dtype=torch.int32)
        args["length"].copy_(d.length)
        args["q"].copy_(torch.randn(d.q.shape))
        d.q = args["q"]
        graph.replay()
        torch.cuda.synchronize()
        got = d.check(got=plan.out)
        # (bits: a length beyond what was filled reads NaN)
        again = hs.tree_attention(**dict(args, out=torch.empty_like(got)))
        assert torch.equal(got.view(torch.int16), other.out.view(torch.int16))
        assert torch.equal(again.view(torch.int16), got.view(torch.int16))


def test_attention_is_the_same_wherever_a_query_stands():
    note("attention positions")
    d = Draft(14, 4, 9, 8, 2, 64, 32, [900, 900, 900, 900], torch.bfloat16)
    for t in (d.q, d.k, d.v, d.table, d.mask):
        t[3] = t[0]
    got = d.check()
    assert torch.equal(got[0], got[3])


def test_attention_far_pages():
    """Offsets beyond 32 bits: a pool of 5 GB of keys."""
    note("attention far pages")
    d = Draft(15, 2, 3, 4, 2, 256, 256, [700, 256], torch.bfloat16)
    args = d.gpu()
    far = 5 * (1 << 30) // (2 * 256 * 256)
    big = hs.PagedCache.empty(far, 2, 256, 256)
    ids = torch.arange(args["cache"].pages, device="cuda")
    to = far - 1 - ids * 5000
    for n, t in big.tensors.items():
        t.view(torch.uint8 if t.dtype == torch.float8_e4m3fn else t.dtype)[to] = args["cache"].tensors[n]
    assert int(to.min()) >= 0 and int(to.max()) * 2 * 65536 > 1 << 32
    d.check(cache=big, table=to.int()[args["table"].long()])


@pytest.mark.parametrize("M,heads,slots", [(1, 1, 1 << 23), (1, 1, (1 << 23) + 5), (20, 2, 1 << 23)])
def test_attention_over_as_many_tokens_as_an_int_counts(M, heads, slots):
    """2^31 - 1 tokens, of pages that a table has many times: the last token, whose score is 200 above the others', is
    there (all others' weight is 2^31 e^-200), and work is cut among the workgroups."""
    note("attention over 2^31 - 1 tokens M=%d slots=%d" % (M, slots))
    dim, page = 32, 256
    code = torch.zeros((2, 1, page, dim), dtype=torch.uint8)
    values = code.transpose(2, 3).contiguous()
    code[1, 0, page - 2] = 0x38   # 1; the last token of the last page but one is the last of all
    values[1, 0, :, page - 2] = torch.arange(1, dim + 1).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
    one = torch.ones((2, 1), device="cuda")
    cache = hs.PagedCache(code.cuda(), values.cuda(), one, one.clone())
    table = torch.zeros((2, slots), dtype=torch.int32, device="cuda")
    table[0, (1 << 23) - 1] = 1
    length = torch.tensor([(1 << 31) - 1, 100], dtype=torch.int32, device="cuda")
    q = torch.full((2, M, heads, dim), 200.0 / dim, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, M, 1, dim), dtype=torch.bfloat16, device="cuda")
    got = hs.tree_attention(q, k, k, cache, table, length, scale=1.0).cpu()
    want = values[1, 0, :, page - 2].view(torch.float8_e4m3fn).to(torch.bfloat16)
    assert torch.equal(got[0], want.expand(got[0].shape)) and torch.all(got[1] == 0)


# ---- hs_cache_append ---------------------------------------------------------------------------------------

def pool(g, pages, kv, page, dim):
    codes = torch.randint(0, 256, (2, pages, kv, page * dim), generator=g).to(torch.uint8)
    scale = torch.exp2(torch.randint(-9, -5, (2, pages, kv), generator=g).float())
    return [codes[0].reshape(pages, kv, page, dim), codes[1].reshape(pages, kv, dim, page), scale[0], scale[1]]


def check_append(state, table, length, k, v, path=None, count=None, gpu=None, **kw):
    """One append to the tensors of `state` and, by the oracle, to their copies: every byte the same (any NaN is NaN)."""
    up = lambda t: None if t is None else t if t.is_cuda else t.cuda()  # noqa: E731
    dev = [up(t.clone()) for t in state] if gpu is None else gpu
    hs.cache_append(hs.PagedCache(*dev), up(table), up(length), up(k), up(v), path=up(path), count=up(count), **kw)
    torch.cuda.synchronize()
    num = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    ref = [t.numpy().copy() for t in state]
    draft.append(*ref, num(table), num(length), k.cpu().double().numpy(), v.cpu().double().numpy(), path=num(path),
                 count=num(count))
    got = [t.cpu().numpy() for t in dev]
    for n in (0, 1):
        same = (got[n] == ref[n]) | (((got[n] & 0x7F) == 0x7F) & ((ref[n] & 0x7F) == 0x7F))
        assert same.all(), (n, np.argwhere(~same)[:4], got[n][~same][:4], ref[n][~same][:4])
    for n in (2, 3):
        assert np.array_equal(got[n], ref[n]), n
    return [torch.from_numpy(t) for t in got]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kv,dim,page,taken,lengths", [
    (1, 32, 32, 1, [0, 1, 31, 32]), (2, 64, 32, 5, [0, 27, 28, 30, 95]), (3, 128, 64, 64, [0, 1, 63, 64, 200]),
    (2, 96, 128, 300, [0, 5, 127, 128]), (1, 256, 256, 257, [0, 255, 256, 3]), (8, 128, 64, 13, [60, 50, 51, 52])])
def test_append_sizes(dtype, kv, dim, page, taken, lengths):
    note("append %s heads=%d dim=%d page=%d taken=%d %s" % (dtype, kv, dim, page, taken, lengths))
    g = torch.Generator().manual_seed(kv * 100 + dim + taken)
    B, slots = len(lengths), -(-(max(lengths) + taken) // page)
    state = pool(g, B * slots + 1, kv, page, dim)
    table = torch.randperm(B * slots + 1, generator=g)[:B * slots].reshape(B, slots).int()
    for spread in (0.01, 1.0, 100.0):  # scales that stay, and that grow
        k = (torch.randn((B, taken, kv, dim), generator=g) * spread).to(dtype)
        v = (torch.randn((B, taken, kv, dim), generator=g) * spread).to(dtype)
        check_append(state, table, torch.tensor(lengths, dtype=torch.int32), k, v)
        count = torch.randint(-1, taken + 2, (B,), generator=g).int()
        check_append(state, table, torch.tensor(lengths, dtype=torch.int32), k, v, count=count)


@pytest.mark.parametrize("kv,dim,page,taken,lengths", [
    (2, 256, 128, 260, [0, 5, 127, 128]), (1, 256, 256, 1, [0, 255, 256]), (1, 128, 256, 130, [200, 3]),
    (2, 256, 64, 64, [63, 0, 33]), (1, 224, 128, 77, [100, 128]), (1, 256, 128, 66, [126, 61, 3]),
    (1, 256, 256, 130, [253, 2]), (3, 160, 256, 255, [1, 2])])
def test_append_large_pages(kv, dim, page, taken, lengths):
    """Workgroups of each size, with pages that are full, begun or ended inside a square."""
    note("append large pages kv=%d dim=%d page=%d taken=%d %s" % (kv, dim, page, taken, lengths))
    g = torch.Generator().manual_seed(dim + page + taken)
    B = len(lengths)
    slots = (max(lengths) + taken + page - 1) // page
    for dtype in (torch.bfloat16, torch.float16):
        state = pool(g, B * slots + 1, kv, page, dim)
        table = torch.randperm(B * slots + 1, generator=g)[:B * slots].reshape(B, slots).int()
        k = torch.randn((B, taken, kv, dim), generator=g).to(dtype) * 3
        v = torch.randn((B, taken, kv, dim), generator=g).to(dtype) * 0.1
        check_append(state, table, torch.tensor(lengths, dtype=torch.int32), k, v)
        v[0, taken // 2, 0, 3] = float("nan")  # the slow way
        check_append(state, table, torch.tensor(lengths, dtype=torch.int32), k, v)


def test_append_paths():
    note("append paths")
    g = torch.Generator().manual_seed(21)
    B, rows, kv, dim, page = 6, 40, 2, 64, 32
    state = pool(g, 20, kv, page, dim)
    table = torch.randperm(20, generator=g)[:18].reshape(6, 3).int()
    k, v = (torch.randn((B, rows, kv, dim), generator=g).to(torch.bfloat16) for _ in range(2))
    path = torch.full((B, 9), -1, dtype=torch.int32)
    path[:, :7] = torch.rand((B, rows), generator=g).argsort(1)[:, :7].sort(1).values.int()
    path[1, 3] = path[1, 2]  # a row twice
    count = torch.tensor([7, 5, 0, 1, 9, 100], dtype=torch.int32)  # (the last two take what is not there: zeros)
    path[5, 0] = 40
    length = torch.tensor([0, 29, 40, 63, 32, 60], dtype=torch.int32)
    check_append(state, table, length, k, v, path=path, count=count)
    wide = torch.full((B, 16), 3, dtype=torch.int32)
    wide[:, :9] = path
    check_append(state, table, length, k, v, path=wide.cuda()[:, :9], count=count)


def test_append_strange_values_and_tables():
    note("append strange values and tables")
    g = torch.Generator().manual_seed(22)
    B, rows, kv, dim, page = 8, 40, 2, 64, 32
    for dtype in (torch.bfloat16, torch.float16):
        state = pool(g, 30, kv, page, dim)
        table = torch.randperm(30, generator=g)[:24].reshape(8, 3).int()
        k, v = (torch.randn((B, rows, kv, dim), generator=g).to(dtype) for _ in range(2))
        k[0], v[0] = 0.0, -0.0
        k[1, 3, 0, 7], v[1, 30, 1, 9] = float("nan"), float("inf")
        k[2], v[2] = float("nan"), -float("inf")
        k[3], v[3] = torch.finfo(dtype).max, torch.finfo(dtype).tiny
        v[4] = 448.0 * 2.0 ** -6   # at the top of a scale, and just above it
        k[4] = (448.0 * 2.0 ** -6) * (1 + 2.0 ** -7)
        table[5, 1], table[6, 0], table[6, 2] = -1, 30, 1 << 30
        length = torch.tensor([5, 0, 20, 0, 0, 3, 20, 90], dtype=torch.int32)  # (the last leaves the table)
        check_append(state, table, length, k, v)
        length = torch.tensor([-1, 96, 1 << 30, -(1 << 31), 64, (1 << 31) - 1, 95, 3], dtype=torch.int32)
        check_append(state, table, length, k, v)


def test_append_scales_that_are_no_powers_of_two():
    note("append other scales")
    g = torch.Generator().manual_seed(23)
    state = pool(g, 9, 2, 32, 64)
    state[2].copy_(torch.rand((9, 2), generator=g) * 0.05)
    state[3].copy_(torch.rand((9, 2), generator=g) * 0.005)
    k, v = (torch.randn((4, 20, 2, 64), generator=g).to(torch.float16) for _ in range(2))
    check_append(state, torch.arange(8).reshape(4, 2).int(), torch.tensor([3, 30, 31, 12], dtype=torch.int32), k, v)


def test_append_step_by_step():
    """Tokens one by one, with strides and another stream, end where the oracle's do; values stay within half a step
    of 8 bits (2^-4 of themselves, or 2^-10 of the page's scale below its normal codes, once for every doubling)."""
    note("append step by step")
    g = torch.Generator().manual_seed(24)
    B, kv, dim, page, n = 2, 2, 64, 32, 70
    qkv = torch.randn((B, n, 8, dim), generator=g) * torch.linspace(0.1, 3.0, n)[None, :, None, None]
    qkv = qkv.to(torch.bfloat16)
    k, v = qkv[:, :, 4:6], qkv[:, :, 6:]
    state = pool(g, 8, kv, page, dim)
    table = torch.tensor([[6, 1, 3], [0, 7, 2]], dtype=torch.int32)
    s = torch.cuda.Stream()
    big = qkv.cuda()
    for t in range(n):
        dev = [x.cuda() for x in state]
        s.wait_stream(torch.cuda.current_stream())
        state = check_append(state, table, torch.tensor([t, t], dtype=torch.int32), big[:, t:t + 1, 4:6],
                             big[:, t:t + 1, 6:], gpu=dev, stream=s if t % 2 else None)
    for b in range(B):
        for t in range(n):
            p, o = int(table[b, t // page]), t % page
            got = draft.VALUES[state[0][p, :, o].numpy()] * state[2][p].numpy()[:, None]
            x = k[b, t].double().numpy()
            assert np.all(np.abs(got - x) <= np.abs(x) * 2.0 ** -4 + state[2][p].numpy()[:, None] * 2.0 ** -9)


def test_append_captured():
    note("append captured")
    g = torch.Generator().manual_seed(25)
    state = pool(g, 9, 2, 32, 64)
    dev = [t.cuda() for t in state]
    k, v = (torch.zeros((2, 6, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, length = torch.arange(8).reshape(2, 4).int().cuda(), torch.zeros(2, dtype=torch.int32, device="cuda")
    count = torch.zeros(2, dtype=torch.int32, device="cuda")
    plan = hs.CacheAppend(hs.PagedCache(*dev), table, length, k, v, count=count)
    plan.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    for i in range(6):
        k.copy_(torch.randn(k.shape, generator=g) * (i + 1))
        v.copy_(torch.randn(k.shape, generator=g) * (6 - i))
        count.copy_(torch.randint(0, 7, (2,), generator=g))
        before = [t.cpu() for t in dev]
        graph.replay()
        torch.cuda.synchronize()
        after = [t.cpu() for t in dev]
        want = check_append(before, table, length, k, v, count=count)
        for a, w in zip(after, want):
            assert torch.equal(a, w), i
        length += count


def test_append_far_pages():
    note("append far pages")
    g = torch.Generator().manual_seed(26)
    far = 5 * (1 << 30) // (2 * 256 * 256)
    big = hs.PagedCache.empty(far, 2, 256, 256)
    to = torch.tensor([far - 1, far - 4000], device="cuda")
    small = pool(g, 2, 2, 256, 256)
    for n, t in zip(big.tensors.values(), small):
        n.view(t.dtype)[to] = t.cuda()
    k, v = (torch.randn((1, 200, 2, 256), generator=g).to(torch.float16) for _ in range(2))
    length = torch.tensor([100], dtype=torch.int32)
    hs.cache_append(big, to.int()[None], length.cuda(), k.cuda(), v.cuda())
    want = check_append(small, torch.tensor([[0, 1]], dtype=torch.int32), length, k, v)
    for n, t in zip(big.tensors.values(), want):
        assert torch.equal(n.view(t.dtype)[to].cpu(), t)


# ---- together ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("mode", [hs.SAMPLE, hs.GREEDY])
def test_rounds_of_a_tree_as_a_program_runs_them(mode):
    """Prompts to the cache; then rounds of growth, the target's attention over the tree, its logits, the verification
    and the accepted nodes' keys and values to the cache. Cache and attention follow a program that keeps every
    accepted token's keys and values; paths follow the oracle."""
    note("rounds mode=%d" % mode)
    g = torch.Generator().manual_seed(41)
    B, W, K, M, depth, V, kv, heads, dim, page = 3, 4, 6, 12, 3, 500, 2, 4, 64, 32
    embed = torch.randn((V, dim), generator=g)
    wq, wk, wv = (torch.randn((dim, n, dim), generator=g) * dim ** -0.5 for n in (heads, kv, kv))
    wo = torch.randn((heads * dim, V), generator=g) * 2.0
    project = lambda t, w: torch.einsum("...d,dhe->...he", embed[t.clamp(min=0).long()], w).to(torch.bfloat16)  # noqa: E731
    cache = hs.PagedCache.empty(16, kv, page, dim)
    table = torch.randperm(16, generator=g)[:15].reshape(B, 5).int().cuda()
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    prompt = torch.randint(0, V, (B, 37), generator=g)
    given = torch.tensor([37, 20, 1], dtype=torch.int32, device="cuda")
    hs.cache_append(cache, table, length, project(prompt, wk).cuda(), project(prompt, wv).cuda(), count=given)
    length += given
    kept = [prompt[b, :int(given[b])].tolist() for b in range(B)]  # tokens in the cache
    root = torch.randint(0, V, (B,), generator=g)
    growth = hs.TreeGrowth(B, depth, W, K, M, device="cuda:0")
    for _ in range(6):
        growth.level(torch.randn((B, 1, V + 4), generator=g).cuda().to(torch.bfloat16), V=V)
        for _ in range(depth - 1):
            growth.level(torch.randn((B, W, V + 4), generator=g).cuda().to(torch.bfloat16), V=V)
        tree_ = growth.tree()
        token = tree_["token"].cpu()
        token[:, 0] = root.int()
        q, k, v = (project(token, w).cuda() for w in (wq, wk, wv))
        out = hs.tree_attention(q, k, v, cache, table, length, mask=tree_["mask"], count=tree_["count"])
        logits = (out.float().reshape(B, M, -1) @ wo.cuda()).to(torch.bfloat16)
        logits = torch.nn.functional.pad(logits, (0, 4))
        u = numbers(g, B, M)
        got = hs.verify(logits, tree_["token"], u.cuda(), parent=tree_["parent"], count=tree_["count"], V=V,
                        mode=mode, depth=depth)
        want = draft.verify(logits[:, :, :V].cpu().double().numpy(), token.numpy(), u.numpy(),
                            parent=tree_["parent"].cpu().numpy(), count=tree_["count"].cpu().numpy(),
                            greedy=mode == hs.GREEDY, depth=depth)
        for n in want:
            assert np.array_equal(got[n].cpu().numpy(), want[n]), n
        # the root's and the accepted nodes' rows join the cache
        hs.cache_append(cache, table, length, k, v, path=got["path"], count=got["length"])
        length += got["length"]
        for b in range(B):
            n = int(got["length"][b])
            kept[b] += token[b, got["path"][b, :n].cpu().long()].tolist()
            root[b] = int(got["token"][b, n - 1])
    assert [len(t) for t in kept] == length.tolist()
    # what the cache holds is what was kept, within the steps of 8 bits (see test_append_step_by_step)
    for b in range(B):
        x = project(torch.tensor(kept[b]), wk).double().numpy()
        for t in range(len(kept[b])):
            p, o = int(table[b, t // page]), t % page
            code = cache.k.view(torch.uint8)[p, :, o].cpu().numpy()
            s = cache.k_scale[p].cpu().numpy()[:, None]
            assert np.all(np.abs(draft.VALUES[code] * s - x[t]) <= np.abs(x[t]) * 2.0 ** -4 + s * 2.0 ** -9)


@pytest.mark.parametrize("mode", [hs.SAMPLE, hs.GREEDY])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rounds_see_and_keep_what_the_cache_should_hold(dtype, mode):
    """As above; in every round the attention is the oracle's over the cache's codes as they are, and in the end keys and
    values are those of the tokens that were kept, so that a round that reads or writes a wrong place is seen."""
    note("rounds, attention and values %s mode=%d" % (dtype, mode))
    g = torch.Generator().manual_seed(43)
    B, W, K, M, depth, V, kv, heads, dim, page = 3, 4, 6, 12, 3, 300, 2, 4, 64, 32
    embed = torch.randn((V, dim), generator=g)
    wq, wk, wv = (torch.randn((dim, n, dim), generator=g) * dim ** -0.5 for n in (heads, kv, kv))
    wo = torch.randn((heads * dim, V), generator=g) * 2.0
    project = lambda t, w: torch.einsum("...d,dhe->...he", embed[t.clamp(min=0).long()], w).to(dtype)  # noqa: E731
    cache = hs.PagedCache.empty(16, kv, page, dim)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(float("nan"))  # what no append has written matters to nobody
    table = torch.randperm(16, generator=g)[:15].reshape(B, 5).int().cuda()
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    prompt = torch.randint(0, V, (B, 37), generator=g)
    given = torch.tensor([37, 20, 1], dtype=torch.int32, device="cuda")
    hs.cache_append(cache, table, length, project(prompt, wk).cuda(), project(prompt, wv).cuda(), count=given)
    length += given
    kept = [prompt[b, :int(given[b])].tolist() for b in range(B)]
    root = torch.randint(0, V, (B,), generator=g)
    growth = hs.TreeGrowth(B, depth, W, K, M, device="cuda:0")
    for _ in range(6):
        growth.level(torch.randn((B, 1, V + 4), generator=g).cuda().to(torch.bfloat16), V=V)
        for _ in range(depth - 1):
            growth.level(torch.randn((B, W, V + 4), generator=g).cuda().to(torch.bfloat16), V=V)
        tree_ = growth.tree()
        token = tree_["token"].cpu()
        token[:, 0] = root.int()
        q, k, v = (project(token, w) for w in (wq, wk, wv))
        out = hs.tree_attention(q.cuda(), k.cuda(), v.cuda(), cache, table, length, mask=tree_["mask"],
                                count=tree_["count"])
        codes = [t.cpu() for t in cache.tensors.values()]
        ref, mean, most = draft.attention(*[t.double().numpy() for t in (q, k, v)], codes[0].view(torch.uint8).numpy(),
                                          codes[1].view(torch.uint8).numpy(), codes[2].numpy(), codes[3].numpy(),
                                          table.cpu().numpy(), length.cpu().numpy(), mask=tree_["mask"].cpu().numpy(),
                                          count=tree_["count"].cpu().numpy(), scale=dim ** -0.5)
        for b in range(B):
            n, a = int(tree_["count"][b]), most[b][..., None]
            rel = 2.0 ** -11 + 2 * (dim + 8) * 2.0 ** -24 * a + 2 * (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -22 * a) + \
                2 * (int(length[b]) + M + 300) * 2.0 ** -24
            tol = HALF[dtype] * np.maximum(np.abs(ref[b]), torch.finfo(dtype).tiny) + rel * mean[b]
            assert n > 1 and np.all((np.abs(out[b].cpu().double().numpy() - ref[b]) <= tol)[:n]), b
        logits = torch.nn.functional.pad((out.float().reshape(B, M, -1) @ wo.cuda()).to(torch.bfloat16), (0, 4))
        got = hs.verify(logits, tree_["token"], numbers(g, B, M).cuda(), parent=tree_["parent"], count=tree_["count"],
                        V=V, mode=mode, depth=depth)
        hs.cache_append(cache, table, length, k.cuda(), v.cuda(), path=got["path"], count=got["length"])
        length += got["length"]
        for b in range(B):
            n = int(got["length"][b])
            kept[b] += token[b, got["path"][b, :n].cpu().long()].tolist()
            root[b] = int(got["token"][b, n - 1])
    assert [len(t) for t in kept] == length.tolist()
    for codes, scale, w in ((cache.k.transpose(2, 3), cache.k_scale, wk), (cache.v, cache.v_scale, wv)):
        codes, scale = codes.contiguous().view(torch.uint8).cpu().numpy(), scale.cpu().numpy()  # [pages][heads][dim][page]
        for b in range(B):
            x = project(torch.tensor(kept[b]), w).double().numpy()
            for t in range(len(kept[b])):
                p, o = int(table[b, t // page]), t % page
                y = draft.VALUES[codes[p, :, :, o]] * scale[p][:, None]
                assert np.all(np.abs(y - x[t]) <= np.abs(x[t]) * 2.0 ** -4 + scale[p][:, None] * 2.0 ** -9), (b, t)
