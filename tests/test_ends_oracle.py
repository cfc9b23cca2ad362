"""CPU pins of the oracle of the operators at a model's two ends."""
import math

import numpy as np

from tests import ends_oracle as o


def test_codes_by_hand():
    x = np.zeros((1, 32))
    x[0, :12] = [6.0, 5.0, 2.5, 3.5, 0.25, 0.75, -0.26, -0.0, 7.9, 1.75, -1.25, 4.99]
    q, s = o.mx4_quantise(x)
    assert s[0, 0] == 127
    v = o.mx4_values(q, s)[0, :12]
    assert v.tolist() == [6.0, 4.0, 2.0, 4.0, 0.0, 1.0, -0.5, 0.0, 6.0, 2.0, -1.0, 4.0]
    assert math.copysign(1, v[7]) == -1
    # 8 begins the next power of two, and every value is its own nearest
    x[0, 8] = 8.0
    assert o.mx4_quantise(x)[1][0, 0] == 128
    every = np.concatenate([o.GRID, -o.GRID, o.GRID, -o.GRID])[None] * 2.0 ** -20
    assert np.array_equal(o.mx4_values(*o.mx4_quantise(every)), every)


def test_nearest_by_brute_force():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((8, 64)) * np.exp2(rng.integers(-30, 30, (8, 1)))
    q, s = o.mx4_quantise(x)
    v = o.mx4_values(q, s).reshape(8, 2, 32)
    b = x.reshape(8, 2, 32)
    unit = np.ldexp(1.0, s.astype(int) - 127)[:, :, None]
    most = np.abs(b).max(2)[:, :, None] / unit
    assert (most >= 4).all() and (most < 8).all()
    all_values = np.concatenate([o.GRID, -o.GRID])
    best = np.abs(b[..., None] / unit[..., None] - all_values).min(-1)
    assert np.allclose(np.abs(b - v) / unit, best, rtol=0, atol=1e-12)


def test_zero_tiny_and_broken_blocks():
    x = np.zeros((1, 128))
    x[0, 32:64] = 2.0 ** -140
    x[0, 70] = math.inf
    x[0, 100], x[0, 101] = math.nan, 1.0
    q, s = o.mx4_quantise(x)
    assert s.tolist() == [[0, 0, 255, 255]]
    assert not q.any() and np.isnan(o.mx4_values(q, s)[0, 64:]).all()


def test_verify_by_hand():
    rows = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1], [0.2, 0.2, 0.6]]))
    drafts = np.log(np.array([[0.25, 0.5, 0.25], [0.8, 0.1, 0.1]]))
    one = np.ones(3)
    # 0.49 * 0.5 < 0.25: accepted; then 0.2 * 0.8 > 0.1: rejected, only token 1 has p > q
    v = o.verify(rows, drafts, [1, 0], [0.49, 0.2], one, 1.0, 1.0)
    assert v.tokens == [1] and list(v.last) == [1]
    # all accepted: the last position's race, by the noise
    v = o.verify(rows, drafts, [0, 1], [0.9, 0.9], np.array([0.2, 5.0, 0.61]), 1.0, 1.0)
    assert v.tokens == [0, 1] and list(v.last) == [0]
    # without the draft's probabilities: accepted with p, and the token itself is out
    # (0.1 / 0.1 is above 0.8 / 1)
    v = o.verify(rows, None, [1, -1], [0.24, 0.0], np.array([0.1, 1.0, 1.0]), 1.0, 1.0)
    assert v.tokens == [1] and list(v.last) == [0]
    v = o.verify(rows, None, [1, -1], [0.26, 0.0], np.array([10.0, 1e-6, 1.0]), 1.0, 1.0)
    assert v.tokens == [] and list(v.last) == [2]
    # greedy, with equal largest logits
    v = o.verify(rows, None, [0, 1], None, None, 1.0, 1.0)
    assert v.tokens == [0, 1] and list(v.last) == [2]
    v = o.verify(np.zeros((3, 3)), None, [0, 2], None, None, 1.0, 1.0)
    assert v.tokens == [0] and list(v.last) == [0]
    assert o.verify(np.full((1, 3), -math.inf), None, [], None, None, 1.0, 1.0).last == {-1: 0.0}


def test_verified_tokens_follow_the_target():
    """Accepting, rejecting and the residual together give the target's distribution."""
    rng = np.random.default_rng(1)
    p, q = rng.dirichlet(np.ones(5)), rng.dirichlet(np.ones(5))
    rows, drafts = np.log(np.stack([p, p])), np.log(q)[None]
    n, seen = 20000, np.zeros(5)
    for _ in range(n):
        d = rng.choice(5, p=q)
        v = o.verify(rows, drafts, [d], [rng.random()], rng.exponential(size=5), 1.0, 1.0)
        seen[v.tokens[0] if v.tokens else list(v.last)[0]] += 1
    # five standard deviations of a count
    assert (np.abs(seen - n * p) < 5 * np.sqrt(n * p * (1 - p))).all()


def test_embedding_gradient_by_hand():
    g, size, count = o.embedding_grad([7, -1, 9, 7, 4], [[1, 2], [9, 9], [3, -4], [5, 6], [8, 8]], 7, 3, 2.0)
    assert g.tolist() == [[12, 16], [0, 0], [6, -8]] and count.tolist() == [2, 0, 1]
    assert size.tolist() == [[12, 16], [0, 0], [6, 8]]
