"""Pins of oracle/draft.py: what comes out of a verification is distributed as the target's own tokens
(summed over a grid of the random numbers), and hand-worked drafts."""
import itertools

import numpy as np
import pytest

from oracle import draft


def grid(n):
    return (np.arange(n) + 0.5) / n


def first_token_law(logits, token, parent, n, T, drafter=None, draws=None):
    """The law of the first token that comes out, over all numbers of nodes 1 .. and of the draw."""
    M, V = logits.shape
    law = np.zeros(V)
    for us in itertools.product(grid(n), repeat=M):
        o = draft.verify(logits[None], np.array([token]), np.array([us]),
                         parent=None if parent is None else np.array([parent]),
                         drafter=None if drafter is None else drafter[None], T=T)
        law[o["token"][0, 0]] += 1.0
    return law / n ** M


@pytest.mark.parametrize("T", [0.7, 1.0])
@pytest.mark.parametrize("token", [[-1, 2, 0], [-1, 2, 2], [-1, 4, 7]])
def test_the_first_token_of_a_tree_is_the_targets(T, token):
    """Two children of the root (the second may repeat the first one's token, or be none)."""
    rng = np.random.default_rng(3)
    z = rng.normal(size=(3, 5))
    n = 40
    law = first_token_law(z, token, [-1, 0, 0], n, T)
    # each of the three numbers lies on a grid of n: its probabilities are off by 1 / n at most
    assert np.abs(law - draft.distribution(z[0], T)).max() <= 3.0 / n


def test_the_first_token_of_a_chain_with_its_drafter_is_the_targets():
    rng = np.random.default_rng(4)
    z, y = rng.normal(size=(2, 4)), rng.normal(size=(1, 4))
    n, T = 200, 0.8
    q = draft.distribution(y[0], T)
    law = sum(q[x] * first_token_law(z, [-1, x], None, n, T, drafter=y) for x in range(4))
    assert np.abs(law - draft.distribution(z[0], T)).max() <= 2.0 / n


def test_all_the_mass_on_the_children_is_always_accepted():
    z = np.full((1, 3, 6), -np.inf)
    z[0, 0, [1, 4]] = [0.3, -0.2]
    z[0, 1:, :] = 0.0
    for u in (0.0, 0.5, 1.0 - 2.0 ** -53):
        o = draft.verify(z, np.array([[-1, 4, 1]]), np.full((1, 3), u), parent=np.array([[-1, 0, 0]]))
        assert o["length"][0] == 2 and o["token"][0, 0] in (1, 4)


def test_greedy_follows_the_argmax():
    z = np.zeros((1, 4, 5))
    z[0, 0, 3] = z[0, 0, 4] = 2.0  # the lower of two
    z[0, 2, 1] = 1.0
    o = draft.verify(z, np.array([[-1, 4, 3, 1]]), None, parent=np.array([[-1, 0, 0, 2]]), greedy=True)
    assert o["path"][0].tolist() == [0, 2, 3, -1] and o["token"][0].tolist() == [3, 1, 0, -1]
    o = draft.verify(z, np.array([[-1, 4, 3, 1]]), None, parent=np.array([[-1, 0, 0, 2]]), greedy=True, depth=1)
    assert o["path"][0].tolist() == [0, 2, -1, -1] and o["token"][0].tolist() == [3, 1, -1, -1]


def test_a_row_without_a_distribution_ends_the_path():
    z = np.zeros((1, 3, 4))
    z[0, 1, 2] = np.nan
    o = draft.verify(z, np.array([[-1, 1, 1]]), np.zeros((1, 3)))
    assert o["path"][0].tolist() == [0, 1, -1] and o["token"][0].tolist() == [1, -1, -1] and o["length"][0] == 2
    o = draft.verify(z, np.array([[-1, 1, 1]]), np.zeros((1, 3)), count=[0])
    assert o["path"][0].tolist() == [-1, -1, -1] and o["length"][0] == 0


# ---- the cache in 8 bits -------------------------------------------------------------------------------------

def test_codes_are_torchs_float8():
    import torch

    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(draft.VALUES, want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.integers(-4, 3, 4000), want[np.isfinite(want)],
                        (want[1:126] + want[2:127]) / 2, [0.0, -0.0, 448.0, -448.0]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    got = draft.encode(x)
    assert np.array_equal(got, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert draft.encode(np.array([1e9, -1e9, np.inf, np.nan])).tolist() == [0x7E, 0xFE, 0x7F, 0x7F]


def test_scales():
    assert draft.least_scale(0.0) == 2.0 ** -40 and draft.least_scale(448.0) == 1.0
    assert draft.least_scale(448.1) == 2.0 and draft.least_scale(224.0) == 0.5 and draft.least_scale(3e38) == 2.0 ** 40


def test_append_then_attend_is_attention_over_the_rows():
    rng = np.random.default_rng(1)
    B, kv, page, dim, n = 2, 2, 32, 8, 40
    k, v = np.zeros((6, kv, page, dim), np.uint8), np.zeros((6, kv, dim, page), np.uint8)
    ks, vs = np.zeros((6, kv), np.float32), np.zeros((6, kv), np.float32)
    table = np.array([[3, 0], [5, 1]])
    x = draft.VALUES[rng.integers(1, 0x60, (2, B, n, kv, dim))]  # values that 8 bits hold
    for i in range(0, n, 10):
        draft.append(k, v, ks, vs, table, [i] * B, x[0, :, i:i + 10], x[1, :, i:i + 10])
    q = rng.normal(size=(B, 1, 4, dim))
    zero = np.zeros((B, 1, kv, dim))
    out, _, _ = draft.attention(q, zero, zero, k, v, ks, vs, table, [n] * B, mask=np.zeros((B, 1), int), scale=0.01)
    for b in range(B):
        for g in range(4):
            s = x[0, b, :, g // 2] @ q[b, 0, g] * 0.01
            w = np.exp(s - s.max())
            assert np.allclose(out[b, 0, g], w @ x[1, b, :, g // 2] / w.sum(), rtol=1e-12)
