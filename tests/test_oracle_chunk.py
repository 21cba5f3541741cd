"""The oracle of steps with several tokens a sequence, pinned to closed forms, invariants and brute force."""
import cmath
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import attention, chunk
from oracle.pages import Model


@pytest.mark.parametrize("interleaved", (False, True))
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, freq, pos = rng.standard_normal((3, 2, 10)), np.array([1.0, 0.25, 1e-3]), [0, 7, 100003]
    y = chunk.rotate(x, pos, freq, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 6:], x[..., 6:])
    for r, p in enumerate(pos):
        for j, f in enumerate(freq):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + 3)
            for h in range(2):
                z = complex(x[r, h, a], x[r, h, b]) * cmath.exp(1j * p * f)
                assert abs(z - complex(y[r, h, a], y[r, h, b])) < 1e-10


def test_scores_depend_on_distances_alone():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 8))
    freq = 10.0 ** -np.arange(4)
    dots = [float((chunk.rotate(q, [p + 5], freq, False) * chunk.rotate(k, [p], freq, False)).sum()) for p in (0, 3, 1000)]
    assert max(dots) - min(dots) < 1e-9


def test_which_keys_are_seen():
    assert chunk.sees(3, 6, 0, 0).tolist() == [1, 1, 1, 1, 0, 0]
    assert chunk.sees(3, 6, 2, 0).tolist() == [0, 0, 1, 1, 0, 0]
    assert chunk.sees(3, 6, 2, 1).tolist() == [1, 0, 1, 1, 0, 0]
    assert chunk.sees(1, 6, 0, 4).tolist() == [1, 1, 1, 1, 0, 0]
    assert not chunk.sees(-1, 6, 0, 0).any()


def test_the_last_row_is_a_decode_step():
    rng = np.random.default_rng(3)
    q, K, V = rng.standard_normal(16), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    out, mean, _ = chunk.attend(q, K, V, 8)
    assert np.allclose(out, attention.attend_one(q, K, V), atol=1e-14) and (mean >= np.abs(out)).all()
    assert np.allclose(chunk.attend(q, K, V, 3)[0], attention.attend_one(q, K[:4], V[:4]), atol=1e-14)
    assert np.allclose(chunk.attend(q, K, V, 8, window=3)[0], attention.attend_one(q, K[6:], V[6:]), atol=1e-14)


def test_caps_and_slopes_by_hand():
    K, V = np.array([[1.0], [2.0]]), np.array([[1.0], [0.0]])
    out = chunk.attend(np.array([3.0]), K, V, 1, scale=1.0, cap=2.0, slope=0.5)[0]
    s = [2 * math.tanh(1.5) - 0.5, 2 * math.tanh(3.0)]
    assert abs(out[0] - math.exp(s[0]) / (math.exp(s[0]) + math.exp(s[1]))) < 1e-15
    assert chunk.attend(np.array([3.0]), K, V, -1)[0].tolist() == [0.0]


def test_probabilities():
    assert chunk.probs([0.0, math.log(3.0)], 1.0).tolist() == pytest.approx([0.25, 0.75])
    assert chunk.probs([0.0, math.log(3.0)], 0.5).tolist() == pytest.approx([0.1, 0.9])
    assert chunk.probs([1.0, 5.0, 5.0], 0).tolist() == [0, 1, 0]
    assert chunk.probs([-math.inf] * 2, 1.0).tolist() == [0, 0]


@pytest.mark.parametrize("certain", (False, True))
def test_verified_tokens_are_drawn_from_the_target(certain):
    """Over a grid of random numbers every token comes as often as the target has it, whatever the draft."""
    p, q = [Fraction(x, 16) for x in (5, 1, 8, 2)], [Fraction(x, 16) for x in ((0, 0, 16, 0) if certain else (2, 6, 4, 4))]
    target = np.array([[float(x) for x in p]] * 2, dtype=np.float32)
    draft = np.array([[float(x) for x in q]], dtype=np.float32)
    came = [Fraction(0)] * 4
    for x in range(4):
        if not q[x]:
            continue
        for u in range(96):
            for w in range(96):
                tokens, a = chunk.verify(target, None if certain else draft, np.array([x]), np.array([(u + .5) / 96, (w + .5) / 96], dtype=np.float32))
                assert tokens[:a] == [x][:a] and (a == 1) == (Fraction(2 * u + 1, 192) * q[x] < p[x])
                came[tokens[0]] += q[x] / 96 ** 2
    assert [float(x) for x in came] == pytest.approx([float(x) for x in p], abs=1 / 64)


def test_weights_that_are_none():
    p = np.array([[0.0, 0.0], [0.5, 0.5]], dtype=np.float32)
    assert chunk.verify(p, None, np.array([1]), np.array([0.5, 0.5], dtype=np.float32)) == ([-1, -1], 0)
    assert chunk.verify(p[1:], None, np.array([], dtype=int), np.array([0.5], dtype=np.float32)) == ([1], 0)
    p = np.array([[0.25, 0.75], [0, 0]], dtype=np.float32)                 # nothing above the draft: the target itself
    assert chunk.verify(p, p[:1], np.array([2]), np.array([0.9, 0.1], dtype=np.float32)) == ([0, -1], 0)


def test_pages_of_shortened_sequences():
    m = Model(8, 4, 3, 4)
    m.extend([0, 1], [10, 5])
    m.shrink([0, 1], [3, 5])
    assert m.lens == [7, 0, 0] and m.table[0] == [0, 1, -1, -1] and m.table[1] == [-1] * 4 and m.refs == [1, 1] + [0] * 6
    m.fork([0], [2])
    m.shrink([0], [5])                                                     # into a shared page
    assert m.status == -3 and m.lens == [7, 0, 7]
    m.status = 0
    m.shrink([0], [3])
    assert m.status == 0 and m.lens[0] == 4 and m.refs[:3] == [2, 0, 1]
    m.shrink([2], [2], row_counts=[6])
    assert m.status == -3
