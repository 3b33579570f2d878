"""The oracle of what surrounds a rollout's steps against examples worked by hand, and its gradient against differences."""
import numpy as np
import pytest

from oracle import steps_oracle as S


def test_adjust_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5, -1.0]])
    out, touched, _ = S.adjust(x, np.array([[0, 1, 1, 3, 9, -1]]), [6], [2], [2.0], [0.25], [0.5], np.array([[4, 2, 4, 7]]), np.array([[9.0, 1.0, -3.0, 5.0]]))
    # 0: in the prompt alone; 1: there and once in the answer; 3: once in the answer; 2 and 4: biases, the last one of 4
    assert out.tolist() == [[1.0, -4.0 - 0.25 - 0.5, 2.0, 0.25 - 0.75, -4.0]] and touched.all()
    out, touched, _ = S.adjust(x, allowed=np.array([[0b01101]], np.uint32), allowed_rows=[0])
    assert out.tolist() == [[2.0, -np.inf, 1.0, 0.5, -np.inf]] and touched.tolist() == [[False, True, False, False, True]]
    out, touched, _ = S.adjust(x, np.array([[0]]), [0], allowed=np.array([[0]], np.uint32), allowed_rows=[3])
    assert (out == x).all() and not touched.any()


def test_distill_by_hand():
    # student (1/2, 1/4, 1/4), teacher (1/4, rest 3/4)
    x = np.log(np.array([[0.5, 0.25, 0.25]]))
    loss, grad, *_ = S.distill(x, np.array([[0, -1]]), np.array([[np.log(0.25), 0.0]]), 1.0, 0.0, True)
    assert loss[0] == pytest.approx(0.25 * np.log(0.5) + 0.75 * np.log(1.5))
    assert grad[0] == pytest.approx([0.25, -0.125, -0.125])  # p - q of the named one, the rest by shares
    loss, grad, *_ = S.distill(x, np.array([[0, -1]]), np.array([[np.log(0.25), 0.0]]), 1.0, 0.0, False)
    assert loss[0] == pytest.approx(0.25 * np.log(0.5)) and grad[0] == pytest.approx([0.25 * 0.5 - 0.25, 0.25 * 0.25, 0.25 * 0.25])
    loss, *_ = S.distill(x, np.array([[0, 0]]), np.array([[np.log(0.25), -0.1]]), 1.0, 1.0, True)  # twice: the first place counts
    assert loss[0] == pytest.approx(0.5 * np.log(2) + 0.5 * np.log(0.5 / 0.75))


@pytest.mark.parametrize("reverse", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_distill_gradient_by_differences(reverse, rest, temperature):
    g = np.random.default_rng(1)
    x, t = g.normal(size=(3, 9)), g.normal(size=(3, 9))
    lq = t - np.log(np.exp(t).sum(1, keepdims=True))
    ids = np.stack([g.permutation(9)[:4] for _ in range(3)])
    lq = np.take_along_axis(lq, ids, 1)
    ids[1, 2], lq[2, 1] = -1, -np.inf
    f = lambda y: S.distill(y, ids, lq, temperature, reverse, rest)[0]  # noqa: E731
    grad = S.distill(x, ids, lq, temperature, reverse, rest)[1]
    h = 1e-6
    for i in range(9):
        d = np.zeros_like(x)
        d[:, i] = h
        assert (f(x + d) - f(x - d)) / (2 * h) == pytest.approx(grad[:, i], abs=1e-8)


def test_fork_by_hand():
    # pages of 4: row 0 has 6 tokens in pages 5, 2; row 1 has 4 in page 7; row 2 has 1 in page 0
    tables = np.array([[5, 2, -1], [7, -1, -1], [0, 3, 3]])
    refs = np.array([1, 0, 1, 0, 0, 1, 0, 1])
    t, n, r, copies = S.fork(tables, [6, 4, 1], [0, 1, 0, 1, -1, 0], refs, 4)
    # the first that goes on as row 0 keeps page 2; the others copy 2 of its tokens to the lowest free pages, row 2's page 0 among them
    assert t.tolist() == [[5, 2, -1], [7, -1, -1], [5, 0, -1], [7, -1, -1], [-1, -1, -1], [5, 1, -1]]
    assert n.tolist() == [6, 4, 6, 4, 0, 6] and r.tolist() == [1, 1, 1, 0, 0, 3, 0, 2] and copies == [(2, 0, 2), (2, 1, 2)]
    # no page left for the second copy: it comes out empty, and page 5 is not counted for it
    t, n, r, copies = S.fork(tables[:2], [6, 4], [0, 1, 0, 0], np.array([9, 0, 1, 9, 9, 1, 9, 1]), 4)
    assert t[3].tolist() == [-1, -1, -1] and n.tolist() == [6, 4, 6, 0] and r.tolist() == [9, 1, 1, 9, 9, 2, 9, 1] and copies == [(2, 1, 2)]


def test_grow_by_hand():
    tables = np.array([[5, 2, -1], [7, -1, -1], [-1, -1, -1]])
    t, n, s, r = S.grow(tables, [6, 4, 0], [1, 3, 9], np.array([0, 0, 1, 0, 0, 1, 0, 1]), 5, 4)
    assert t.tolist() == [[5, 2, -1], [7, 0, -1], [1, 3, -1]] and n.tolist() == [7, 7, 5] and r.tolist() == [1, 1, 1, 1, 0, 1, 0, 1]
    assert s.tolist() == [[10, -1, -1, -1, -1], [0, 1, 2, -1, -1], [4, 5, 6, 7, 12]]
    # one page is left, and the second row wants two: it stays, the third cannot have the page either, the fourth needs none
    t, n, s, r = S.grow(np.array([[5, -1], [-1, -1], [-1, -1], [2, -1]]), [4, 0, 0, 1], [1, 5, 1, 2], np.array([1, 0, 1, 0, 1, 1]), 5, 4)
    assert t.tolist() == [[5, 1], [-1, -1], [-1, -1], [2, -1]] and n.tolist() == [5, 0, 0, 3] and r.tolist() == [1, 1, 1, 0, 1, 1]
    assert s[3].tolist() == [9, 10, -1, -1, -1] and (s[1:3] == -1).all()


def test_compact_by_hand():
    (t,), r, places, n, moves = S.compact(np.array([0, 3, 0, 1, 0, 2, 1]), [np.array([[6, 1, -1], [5, 3, 99]])])
    assert n == 4 and places.tolist() == [-1, 1, -1, 3, -1, 0, 2] and r.tolist() == [2, 3, 1, 1, 0, 0, 0]
    assert t.tolist() == [[2, 1, -1], [0, 3, 99]] and moves == [(5, 0), (6, 2)]
