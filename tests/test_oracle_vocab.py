"""Pins of oracle/vocab.py (CPU): the definitions against the mathematics."""

import math

import numpy as np
import pytest

from oracle import vocab


def test_embedding_gradient_is_the_adjoint_of_the_lookup():
    rng = np.random.default_rng(0)
    V, d, T = 11, 5, 40
    tokens, seq = rng.integers(0, V, T), rng.integers(-1, 3, T)
    table, dx = rng.standard_normal((V, d)), rng.standard_normal((T, d))
    left = (vocab.embed(table, tokens, seq, 0.7) * dx).sum()
    right = (table * vocab.embed_backward(dx, tokens, seq, V, 0.7)).sum()
    assert abs(left - right) < 1e-12
    assert np.isnan(vocab.embed(table, [V], [0])).all()


def test_draw_by_hand():
    w = np.array([0.0, 1.0, 0.0, 3.0, 0.0])
    assert [vocab.draw(w, u) for u in (0.0, 0.2499, 0.25, 0.99, 1.0)] == [1, 1, 3, 3, 3]


@pytest.mark.parametrize("drafted", [True, False])
def test_emitted_tokens_follow_the_policy(drafted):
    """Integrated over its random numbers, the first emitted token is distributed as the
    policy, whatever the draft: with sampled drafts, weighting each draft by its q."""
    rng = np.random.default_rng(4)
    V, n = 5, 400
    z, zd = rng.standard_normal((2, V)), rng.standard_normal((1, V)) * 2
    p, q = vocab.distribution(z[0]), vocab.distribution(zd[0])
    grid = (np.arange(n) + 0.5) / n
    got = np.zeros(V)
    for x in range(V):
        weight = q[x] if drafted else 1.0 / V
        for u0 in grid:
            first = vocab.verify(z, zd if drafted else None, [x], 1, [u0, 0.3])[0][0]
            if first == x:
                got[x] += weight / n
            else:  # rejected: integrate the draw
                for u1 in grid[::16]:
                    v = vocab.verify(z, zd if drafted else None, [x], 1, [u0, u1])[0][0]
                    got[v] += weight / n / len(grid[::16])
                    if not drafted:
                        assert v != x
    # a midpoint rule of n and n / 16 points: each of V borders moves by less than a cell
    assert np.abs(got - p).max() < 2.0 * V * 16 / n


def test_no_distribution():
    z = np.zeros((2, 4))
    z[1, 2] = np.nan
    assert vocab.distribution(z[1]) is None
    assert vocab.distribution([-np.inf] * 3) is None
    tokens, logp = vocab.verify(z, None, [1], 1, [0.0, 0.5])
    assert tokens == [1, -1] and logp[0] == math.log(0.25) and math.isnan(logp[1])


@pytest.mark.parametrize("use_mass", [True, False])
def test_distillation_gradient_by_differences(use_mass):
    rng = np.random.default_rng(9)
    T, V, K = 6, 9, 4
    z = rng.standard_normal((T, V))
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    ids[1, 2:] = -1
    ids[2, 1] = ids[2, 0]
    seq, seq_len = np.array([0, 0, 1, 1, -1, 1]), np.array([3, 5])
    lt = rng.standard_normal((T, K)) + 2
    mass = np.log(np.exp(lt / 1.5).sum(1)) + 0.2 if use_mass else None

    def loss(x):
        return vocab.distill(x, ids, lt, mass, seq, seq_len, 2, 1.5, 0.3)[1]

    dz = vocab.distill(z, ids, lt, mass, seq, seq_len, 2, 1.5, 0.3)[3]
    h = 1e-5
    for t in range(T):
        for v in range(V):
            a, b = z.copy(), z.copy()
            a[t, v] += h
            b[t, v] -= h
            assert abs((loss(a) - loss(b)) / (2 * h) - dz[t, v]) < 1e-9
    assert np.abs(dz.sum(1)).max() < 1e-15  # a softmax's gradient


def test_distilling_the_policy_itself_is_zero():
    rng = np.random.default_rng(2)
    z = rng.standard_normal((3, 7))
    ids = np.tile(np.arange(7), (3, 1))
    kl, loss, stats, dz = vocab.distill(z, ids, z, None, [0, 0, 0], [3], 1)
    assert np.abs(kl).max() < 1e-15 and np.abs(dz).max() < 1e-16 and stats[0] == 3
