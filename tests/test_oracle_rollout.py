"""Pins of the rollout oracle: small cases by hand, identities, and the gradient against differences."""
import numpy as np
import pytest

from oracle import rollout_oracle as R


def test_rotation_by_hand_and_its_length():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    cos, sin = np.array([[9.0, 9.0], [0.0, 0.6]]), np.array([[9.0, 9.0], [1.0, 0.8]])
    got, _ = R.rotate(x, np.array([1]), cos, sin, False)            # pairs (1, 3), (2, 4)
    assert np.allclose(got, [[[-3.0, 2 * .6 - 4 * .8, 1.0, 4 * .6 + 2 * .8, 5.0]]])
    got, _ = R.rotate(x, np.array([1]), cos, sin, True)             # pairs (1, 2), (3, 4)
    assert np.allclose(got, [[[-2.0, 1.0, 3 * .6 - 4 * .8, 4 * .6 + 3 * .8, 5.0]]])


def test_scores_of_rotated_pairs_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 8))
    at = np.arange(40)[:, None] * 100.0 ** (-np.arange(4) / 4)
    turn = lambda x, p: R.rotate(x, np.array([p]), np.cos(at), np.sin(at), False)[0].ravel()  # noqa: E731
    assert np.isclose(turn(q, 30) @ turn(k, 21), turn(q, 9) @ turn(k, 0))


def test_attention_by_hand():
    # one KV head, pages of 4 tokens; the prompt is page 2 (3 tokens), the answer page 0 (1 token)
    k, v = np.zeros((3, 1, 4, 1)), np.zeros((3, 1, 4, 1))
    k[2, 0, :, 0], v[2, 0, :, 0] = [0, np.log(2), 0, 1e9], [1, 2, 3, 1e9]
    k[0, 0, :, 0], v[0, 0, :, 0] = [np.log(4), 1e9, 1e9, 1e9], [5, 1e9, 1e9, 1e9]
    q = np.ones((1, 1, 1))
    out, lse, *_ = R.attend(q, k, v, [1], [[0]], [0, 1], [3], [[2]], 1.0)
    assert np.isclose(out[0, 0, 0], (1 + 2 * 2 + 3 + 4 * 5) / 8) and np.isclose(lse[0, 0], np.log(8))
    out, lse, *_ = R.attend(q, k, v, [0], [[0]], None, None, None, 1.0)
    assert out[0, 0, 0] == 0 and lse[0, 0] == -np.inf


def test_logprobs_by_hand():
    x = np.log(np.array([[1.0, 2.0, 5.0], [4.0, 4.0, 8.0]]))
    lp, ent, lse, _, _ = R.logprobs(x, np.array([1, 5]), 1.0)
    assert np.allclose(lp, [np.log(.25), 0]) and np.allclose(lse, [np.log(8), 0])
    assert np.isclose(ent[0], -(.125 * np.log(.125) + .25 * np.log(.25) + .625 * np.log(.625))) and ent[1] == 0
    lp, ent, lse, _, _ = R.logprobs(np.array([[-np.inf, -np.inf], [-np.inf, 3.0]]), np.array([0, 0]), 2.0)
    assert lse.tolist() == [-np.inf, 1.5] and lp.tolist() == [-np.inf, -np.inf] and ent.tolist() == [0, 0]
    assert R.top_ids(np.array([[1.0, 3.0, 3.0, -0.0, 0.0]]), 5).tolist() == [[1, 2, 0, 3, 4]]


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_gradient_against_differences(temperature):
    rng = np.random.default_rng(1)
    x, t = 2 * rng.standard_normal((4, 9)), np.array([3, 0, -100, 8])
    g, h = rng.standard_normal((2, 4))
    x[3, 2] = -np.inf

    def value(x):
        lp, ent, *_ = R.logprobs(x, t, temperature)
        return (g * lp + h * ent).sum()

    got, *_ = R.logprobs_back(x, t, temperature, g, h)
    step = 1e-5
    for r in range(4):
        for j in range(9):
            if x[r, j] == -np.inf:
                assert got[r, j] == 0
                continue
            up, down = x.copy(), x.copy()
            up[r, j] += step
            down[r, j] -= step
            # central difference: error step^2 / 6 * third derivative (below 50 here) + rounding 1e-16 / step
            assert abs((value(up) - value(down)) / (2 * step) - got[r, j]) < 50 * step ** 2 + 1e-9
