"""Pins of the attention sublayer's float64 oracle on the CPU: hand-worked
values, invariants, differences for the gradients."""
import numpy as np
import pytest

from oracle import attn_oracle as A


def test_rotation_by_hand():
    # theta = 1: every pair turns by p radians; a quarter turn swaps the pair
    table = np.array([[1.0, 0.0], [0.0, 1.0]])          # angles 0 and pi/2
    x = np.array([[[3.0, 4.0]], [[3.0, 4.0]]])
    y = A.norm_rope(x, pos=[0, 1], table=table, eps=None)
    assert np.array_equal(y, [[[3.0, 4.0]], [[-4.0, 3.0]]])
    x4 = np.arange(1.0, 5.0).reshape(1, 1, 4)
    t4 = np.array([[0.0, 1.0, 1.0, 0.0]])               # first pair a quarter turn, second none
    assert np.array_equal(A.norm_rope(x4, pos=[0], table=t4, eps=None, style="halves"), [[[-3, 2, 1, 4]]])
    assert np.array_equal(A.norm_rope(x4, pos=[0], table=t4, eps=None, style="pairs"), [[[-2, 1, 3, 4]]])
    # a table narrower than the head leaves the rest as it is
    assert np.array_equal(A.norm_rope(x4, pos=[1], table=table, eps=None), [[[-2, 1, 3, 4]]])


def test_table_values():
    t = A.rope_table(3, 4, 100.0)
    assert np.allclose(t[2], [np.cos(2), np.cos(0.2), np.sin(2), np.sin(0.2)], atol=1e-15)


def test_norm_by_hand():
    x = np.array([[[3.0, 4.0]]])                        # mean square 12.5
    assert np.allclose(A.norm_rope(x, eps=0.0), x / np.sqrt(12.5), atol=1e-15)
    assert np.allclose(A.norm_rope(x, w=np.array([2.0, 0.5]), eps=3.5), x / 4 * [2.0, 0.5], atol=1e-15)


@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_rotation_keeps_inner_products_of_equal_distance(style):
    r = np.random.default_rng(0)
    table = A.rope_table(50, 16, 10.0)
    q, k = r.standard_normal((1, 1, 16)), r.standard_normal((1, 1, 16))
    f = lambda x, p: A.norm_rope(x, pos=[p], table=table, eps=None, style=style)[0, 0]  # noqa: E731
    assert abs(f(q, 40) @ f(k, 33) - f(q, 7) @ f(k, 0)) < 1e-12


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("eps", [None, 1e-6, 0.3])
@pytest.mark.parametrize("R", [0, 4, 6])
def test_gradients_against_differences(style, eps, R):
    r = np.random.default_rng(R)
    x, gy = r.standard_normal((5, 2, 6)), r.standard_normal((5, 2, 6))
    w = None if eps is None else r.standard_normal(6)
    table, pos = A.rope_table(9, R, 50.0), [0, 8, 3, 3, 1]
    f = lambda x, w: (A.norm_rope(x, w, pos, table, eps, style) * gy).sum()  # noqa: E731
    gx, gw = A.norm_rope_backward(x, gy, w, pos, table, eps, style)
    h = 1e-6

    def difference(a, e, call):
        hi, lo = a.copy(), a.copy()
        hi.flat[e] += h
        lo.flat[e] -= h
        return (call(hi) - call(lo)) / (2 * h)
    for e in range(x.size):
        assert abs(difference(x, e, lambda v: f(v, w)) - gx.flat[e]) < 1e-8
    for e in range(0 if w is None else w.size):
        assert abs(difference(w, e, lambda v: f(x, v)) - gw.flat[e]) < 1e-8


def test_attention_of_one_key_and_of_equal_scores():
    r = np.random.default_rng(1)
    V = r.standard_normal((2, 1, 3, 4))                  # two pages of three
    K = np.zeros_like(V)
    O, lse, _ = A.paged_attention(r.standard_normal((3, 2, 4)), K, V, [[1, 0]], [0, 3], [5], 1.0)
    # positions 2, 3, 4 see the means of 3, 4, 5 values in page order 1, 0
    v = np.concatenate([V[1, 0], V[0, 0]])
    for i in range(3):
        assert np.allclose(O[i], v[:3 + i].mean(0), atol=1e-15)
        assert np.allclose(lse[i], np.log(3 + i), atol=1e-15)


def test_attention_by_hand():
    # scores ln 1 and ln 3: weights 1/4 and 3/4
    K = np.array([[[[0.0], [np.log(3)]]]])
    V = np.array([[[[8.0], [4.0]]]])
    O, lse, M = A.paged_attention(np.ones((1, 1, 1)), K, -V, [[0]], [0, 1], [2], 1.0)
    assert np.allclose([O[0, 0, 0], M[0, 0, 0], lse[0, 0]], [-5.0, 5.0, np.log(4)], atol=1e-15)


def test_rows_that_see_nothing_and_padding():
    K = V = np.ones((1, 1, 4, 2))
    O, lse, _ = A.paged_attention(np.ones((4, 1, 2)), K, V, [[0], [0]], [1, 3, 3], [1, 3], 1.0)
    assert np.isnan(O[0]).all() and np.isnan(O[3]).all()
    assert (O[1] == 0).all() and lse[1, 0] == -np.inf and (O[2] == 1).all()
