"""The 64-bit forms of drafted decoding against hand-made cases and independent
statements of the same thing (CPU only)."""
import math

import numpy as np
import pytest

from oracle import draft_oracle as do
from oracle import paged_oracle as po


def test_turns_of_far_positions():
    assert do.turn(0, 0.5) == 0.0
    assert abs(do.turn(7, 1.0) - (7 / (2 * math.pi) - 1)) < 1e-15
    assert abs(do.turn(-7, 1.0) - (2 - 7 / (2 * math.pi))) < 1e-15
    # sin by the standard library, whose argument reduction is exact
    assert abs(math.sin(2 * math.pi * do.turn(2 ** 31 - 1, 1.0)) - math.sin(2.0 ** 31 - 1)) < 1e-14


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_differences(interleaved):
    """Rotated queries and keys have products that depend on the distance only."""
    rng = np.random.default_rng(0)
    x, y = rng.normal(size=(2, 1, 3, 64))
    inv = 1e4 ** (-np.arange(16) / 16)
    def dot(a, b):
        q, k = (do.norm_rope(z, [p], inv, None, 0, interleaved) for z, p in ((x, a), (y, b)))
        assert np.allclose((q ** 2).sum(-1), (x ** 2).sum(-1))
        return (q * k).sum(-1)
    assert np.allclose(dot(1000, 990), dot(14, 4))
    assert not np.allclose(dot(1000, 990), dot(14, 5))


def test_norm_by_hand():
    y = do.norm_rope(np.array([[[3.0, 4.0]]]), [0], None, [1.0, 2.0], 0.0, False)
    assert np.allclose(y, [[[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]]])


def test_ancestors():
    parent = [-1, 0, 0, 1, 3, -1, 5, 9, 2]
    assert do.ancestors(parent, 4) == [4, 3, 1, 0] and do.ancestors(parent, 8) == [8, 2, 0]
    assert do.ancestors(parent, 6) == [6, 5] and do.ancestors(parent, 7) == [7]


def test_a_chain_is_the_causal_block():
    rng = np.random.default_rng(1)
    q, kb, vb = rng.normal(size=(1, 5, 4, 64)), rng.normal(size=(1, 5, 2, 64)), rng.normal(size=(1, 5, 2, 64))
    c, s = rng.integers(0, 120, (3, 2, 16, 64)).astype(np.uint8), np.ones((3, 2))
    args = (q, c, c, s, s, np.array([[2, 0, -1]]), [20], kb, vb)
    a = do.tree_attention(*args, np.array([[-1, 0, 1, 2, 3]]))
    b = po.block_attention(*args, n_causal=5)
    for x, y in zip(a, b):
        assert np.allclose(x, y, rtol=1e-13)


@pytest.mark.parametrize("drawn", [True, False])
def test_verified_tokens_have_the_targets_distribution(drawn):
    """The first token that comes out of a node with two children is distributed as p."""
    rng = np.random.default_rng(2)
    V, n = 5, 40000
    target, draft = rng.normal(size=(3, V)), rng.normal(size=(3, V))
    p, q = (np.exp(z[0]) / np.exp(z[0]).sum() for z in (target, draft))
    seen = np.zeros(V)
    for _ in range(n):
        x = rng.choice(V, size=2, p=q) if drawn else np.array([1, 3])
        _, tokens, _, _ = do.verify(target, draft if drawn else None, [-1, 0, 0], [0, *x], rng.random(3),
                                    rng.gumbel(size=V), 1.0)
        seen[tokens[0]] += 1
    assert np.abs(seen / n - p).max() < 5 * math.sqrt(0.25 / n)


def test_verification_by_hand():
    big = 30.0
    z = np.zeros((4, 3))
    z[0, 2] = z[1, 1] = z[2, 0] = z[3, 1] = big
    # greedy: 0 -> child 2 (token 2) -> no child with token 0
    path, tokens, logprob, _ = do.verify(z, None, [-1, 0, 0, 2], [9, 1, 2, 1], None, None, 0)
    assert path == [0, 2] and tokens == [2, 0] and max(map(abs, logprob)) < 1e-12
    # ties go to the lowest index, in a row of nothing all are alike
    assert do.verify(np.zeros((1, 4)), None, [-1], [0], None, None, 0)[1] == [0]
    none = np.full((2, 3), -np.inf)
    assert do.verify(none, None, [-1, 0], [0, 1], [0, 0.4], np.zeros(3), 1.0)[:2] == ([0], [0])
    assert do.verify(none, None, [-1, 0], [0, 1], [0, 0.3], np.zeros(3), 1.0)[:2] == ([0, 1], [1, 0])
    assert do.verify(none, None, [-1, 0], [0, 0], None, None, 0)[:2] == ([0, 1], [0, 0])
    # equal distributions: accepted below 1, and where a token is refused all the same, p stays
    z = np.log([[0.25, 0.75], [0.5, 0.5]])
    assert do.verify(z, z, [-1, 0], [0, 0], [0, 0.999999], np.array([9.0, 0.0]), 1.0)[0] == [0, 1]
    path, tokens, _, _ = do.verify(z, z, [-1, 0], [0, 0], [0, 1.0], np.array([9.0, 0.0]), 1.0)
    assert path == [0] and tokens == [0]


def test_append_of_a_path_is_the_append_of_its_nodes():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(2, 4, 1, 64))
    codes, scale = np.zeros((4, 1, 16, 64), np.uint8), np.zeros((4, 1), np.float32)
    a = do.append_path(x, np.array([[0, 2, 3, -1], [0, 1, -1, -1]]), [0, 3, 5], [14, 15, 32, 16, 17, -1, -1, -1], codes, scale, 16)
    b = po.cache_append(x.reshape(8, 1, 64)[[0, 2, 3, 4, 5]], [14, 15, 32, 16, 17], codes, scale, 16)
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
