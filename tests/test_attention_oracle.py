"""The attention oracle against what its definition fixes by hand (no GPU)."""
import math

import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc

rng = np.random.default_rng(3)


def test_hand_example_of_two_keys():
    # q.k = 0 and ln 3: weights 1/4 and 3/4
    k = np.array([[[0.0, 0.0]], [[1.0, 0.0]]])
    q = np.array([[[math.log(3.0), 5.0]]])
    v = np.array([[[4.0, 0.0]], [[8.0, 1.0]]])
    out, lse, sums, *_ = orc.attend(q, k, v, 1.0)
    assert np.allclose(out[0, 0], [7.0, 0.75]) and np.isclose(lse[0, 0], math.log(4.0)) and np.allclose(sums[:, 0], [0.25, 0.75])


def test_zero_queries_average_what_they_see():
    n, new = 7, 3
    v = rng.standard_normal((n, 2, 4))
    out, lse, sums, *_ = orc.attend(np.zeros((new, 4, 4)), rng.standard_normal((n, 2, 4)), v, 0.5)
    for t in range(new):
        assert np.allclose(out[t, 1], v[:n - new + t + 1, 0].mean(0)) and np.isclose(lse[t, 3], math.log(n - new + t + 1))
    assert np.isclose(sums.sum(), new * 4)


def test_cap_and_bias_by_hand():
    k, q = np.array([[1.0], [2.0], [3.0]]), np.array([[2.0]])
    s = orc.scores(q, k, 0.5, cap=1.5, slope=0.25)
    want = [1.5 * math.tanh(x / 1.5) - 0.25 * away for x, away in ((1, 2), (2, 1), (3, 0))]
    assert np.allclose(s[0], want)
    assert np.allclose(orc.scores(q, k, 0.5, cap=1e9), orc.scores(q, k, 0.5))
    assert np.allclose(orc.scores(q, k, 0.5, slope=1.0, position=[5, 9, 10])[0], [1 - 5, 2 - 1, 3])


def test_what_is_seen():
    # causal, window of two, prefix of one, two documents
    assert orc.seen(4, 2).tolist() == [[True, True, True, False], [True] * 4]
    assert orc.seen(4, 2, window=2).tolist() == [[False, True, True, False], [False, False, True, True]]
    assert orc.seen(4, 2, window=2, prefix=1).tolist() == [[True, True, True, False], [True, False, True, True]]
    assert orc.seen(4, 3, prefix=3).tolist() == [[True] * 3 + [False]] * 2 + [[True] * 4]
    assert orc.seen(4, 4, doc=[0, 0, 1, -1]).tolist() == [[True, False, False, False], [True, True, False, False],
                                                          [False, False, True, False], [False] * 4]
    assert orc.seen(3, 1, window=2, position=[0, 8, 9]).tolist() == [[False, True, True]]
    assert orc.seen(2, 1, exists=[False, True]).tolist() == [[False, True]]
    assert orc.seen(1, 2).tolist() == [[False], [True]] and orc.seen(0, 1).shape == (1, 0)


def test_a_row_that_sees_nothing():
    out, lse, sums, *_ = orc.attend(np.ones((1, 1, 2)), np.full((3, 1, 2), np.nan), np.full((3, 1, 2), np.nan), 1.0, exists=[False] * 3)
    assert not out.any() and lse[0, 0] == -np.inf and not sums.any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_norms_and_depends_on_differences(interleaved):
    d, pairs = 10, 4
    freq = 0.3 ** np.arange(pairs)
    angle = np.arange(50)[:, None] * freq
    x, y = rng.standard_normal((1, 1, d)), rng.standard_normal((1, 1, d))
    turn = lambda z, p: orc.rotate(z, np.cos(angle), np.sin(angle), np.array([[p]]), [pairs], interleaved)[0, 0]  # noqa: E731
    assert np.isclose(np.linalg.norm(turn(x, 17)), np.linalg.norm(x)) and np.allclose(turn(x, 0), x[0, 0])
    assert np.isclose(turn(x, 31) @ turn(y, 24), turn(x, 12) @ turn(y, 5))
    assert np.array_equal(turn(x, 9)[2 * pairs:], x[0, 0, 2 * pairs:])


def test_rotation_by_a_quarter_and_its_axes():
    cos, sin = np.array([[1.0, 1.0], [0.0, 0.0]]), np.array([[0.0, 0.0], [1.0, 1.0]])
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    pos = np.array([[1], [0]])                         # axis 0 turned by a quarter, axis 1 not at all
    assert np.allclose(orc.rotate(x, cos, sin, pos, [1, 1])[0, 0], [-3, 2, 1, 4])
    assert np.allclose(orc.rotate(x, cos, sin, pos, [1, 1], interleaved=True)[0, 0], [-2, 1, 3, 4])


def test_kept_by_brute_force():
    w = np.array([[1, 0], [5, 0], [2, 1], [0, 3], [0.5, 0], [9, 0]], np.float32)
    assert orc.kept(w, 3).tolist() == [1, 2, 5]        # 3 and 3: the lower index
    assert orc.kept(w, 4).tolist() == [1, 2, 3, 5]
    assert orc.kept(w, 3, sinks=1, recent=1).tolist() == [0, 1, 5]
    assert orc.kept(w, 3, exists=[True, False, True, True, True, False]).tolist() == [0, 2, 3]
    assert orc.kept(w, 9).tolist() == list(range(6)) and orc.kept(w, 0).tolist() == []
    assert orc.kept(np.array([[np.nan], [-1.0], [-np.inf]], np.float32), 2).tolist() == [0, 1]
