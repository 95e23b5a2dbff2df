"""Pins of the cross attention's and the recurrence's oracles: closed forms,
symmetries, and gradients against central differences."""
import numpy as np
import pytest

import oracle.cross_oracle as X
import oracle.recur_oracle as R


def _rng(seed=0):
    return np.random.default_rng(seed)


def test_one_state_is_returned():
    r = _rng()
    q, k, v = r.standard_normal((5, 4)), r.standard_normal((1, 4)), r.standard_normal((1, 4))
    out, lse, p = X.cross_head(q, k, v, 0.7)
    np.testing.assert_allclose(out, np.repeat(v, 5, 0), rtol=1e-14)
    np.testing.assert_allclose(lse, 0.7 * (q @ k.T)[:, 0], rtol=1e-12)


def test_no_state_gives_zero():
    out, lse, _ = X.cross_head(np.ones((3, 4)), np.zeros((0, 4)), np.zeros((0, 4)), 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_equal_scores_average():
    r = _rng(1)
    v = r.standard_normal((7, 4))
    out, lse, _ = X.cross_head(np.zeros((2, 4)), r.standard_normal((7, 4)), v, 1.0)
    np.testing.assert_allclose(out, np.repeat(v.mean(0)[None], 2, 0), rtol=1e-13)
    np.testing.assert_allclose(lse, np.log(7), rtol=1e-14)


def test_order_of_states_and_masks():
    r = _rng(2)
    q, k, v = r.standard_normal((6, 4, 8)), r.standard_normal((9, 2, 8)), r.standard_normal((9, 2, 8))
    seen = r.random(9) < 0.6
    out, lse = X.cross_sequence(q, k, v, seen, 0.5)
    at = r.permutation(9)
    out2, lse2 = X.cross_sequence(q, k[at], v[at], seen[at], 0.5)
    np.testing.assert_allclose(out, out2, rtol=1e-12)
    np.testing.assert_allclose(lse, lse2, rtol=1e-12)
    k[~seen], v[~seen] = np.nan, np.inf
    np.testing.assert_array_equal(X.cross_sequence(q, k, v, seen, 0.5)[0], out)


def _difference(fn, x, dy, h=1e-6):
    """The gradient of sum(fn(x) dy) by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = (fn(x) * dy).sum()
        x[i] = keep - h
        down = (fn(x) * dy).sum()
        x[i] = keep
        g[i] = (up - down) / (2 * h)
    return g


def test_cross_gradients_against_differences():
    r = _rng(3)
    q, k, v = r.standard_normal((3, 4, 4)), r.standard_normal((5, 2, 4)), r.standard_normal((5, 2, 4))
    seen = np.array([True, False, True, True, True])
    do = r.standard_normal(q.shape)
    _, _, dq, dk, dv = X.cross_sequence(q, k, v, seen, 0.8, do)
    run = lambda q, k, v: X.cross_sequence(q, k, v, seen, 0.8)[0]  # noqa: E731
    np.testing.assert_allclose(dq, _difference(lambda x: run(x, k, v), q, do), atol=2e-9)
    np.testing.assert_allclose(dk, _difference(lambda x: run(q, x, v), k, do), atol=2e-9)
    np.testing.assert_allclose(dv, _difference(lambda x: run(q, k, x), v, do), atol=2e-9)


@pytest.mark.parametrize("reverse", [False, True])
def test_constant_decay_is_a_geometric_sum(reverse):
    a, L = 0.9, 12
    x, g = np.ones((L, 1)), np.full((L, 1), np.log(a))
    out, h = R.recur_sequence(x, g, "log", np.array([2.0]), reverse)
    n = np.arange(1, L + 1)
    want = a ** n * 2.0 + (1 - a ** n) / (1 - a)
    np.testing.assert_allclose(out[:, 0], want[::-1] if reverse else want, rtol=1e-13)
    np.testing.assert_allclose(h[0], want[-1], rtol=1e-13)


@pytest.mark.parametrize("gate", ["log", "logit", "norm"])
def test_recurrence_in_two_parts_and_reversed(gate):
    r = _rng(4)
    x, g, h = r.standard_normal((11, 3)), -np.abs(r.standard_normal((11, 3))), r.standard_normal(3)
    out, last = R.recur_sequence(x, g, gate, h)
    a, mid = R.recur_sequence(x[:4], g[:4], gate, h)
    b, end = R.recur_sequence(x[4:], g[4:], gate, mid)
    np.testing.assert_allclose(out, np.concatenate([a, b]), rtol=1e-14)
    np.testing.assert_allclose(last, end, rtol=1e-14)
    back, _ = R.recur_sequence(x[::-1], g[::-1], gate, h, reverse=True)
    np.testing.assert_allclose(back[::-1], out, rtol=1e-14)


def test_norm_keeps_the_variance():
    """With independent inputs of variance 1 the state's variance stays 1."""
    r = _rng(5)
    x, g = r.standard_normal((400, 4000)), np.full((400, 4000), 1.5)
    out, _ = R.recur_sequence(x, g, "norm", r.standard_normal(4000))
    assert abs(out[-1].var() - 1) < 5 * np.sqrt(2 / 4000)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("gate", ["log", "logit", "norm"])
def test_recurrence_gradients_against_differences(gate, reverse):
    r = _rng(6)
    x, g, h = r.standard_normal((6, 2)), -np.abs(r.standard_normal((6, 2))), r.standard_normal(2)
    do, dS = r.standard_normal((6, 2)), r.standard_normal(2)
    both = np.concatenate([do, dS[None]])
    run = lambda x, g, h: np.concatenate([o if o.ndim == 2 else o[None] for o in R.recur_sequence(x, g, gate, h, reverse)])  # noqa: E731
    dx, dg, dh = R.recur_sequence_backward(do, dS, x, g, gate, h, reverse)
    np.testing.assert_allclose(dx, _difference(lambda z: run(z, g, h), x, both), atol=2e-9)
    np.testing.assert_allclose(dg, _difference(lambda z: run(x, z, h), g, both), atol=2e-9)
    np.testing.assert_allclose(dh, _difference(lambda z: run(x, g, z), h, both), atol=2e-9)


def test_a_reset_forgets():
    x, g = np.array([[1.0], [2.0], [3.0]]), np.array([[0.0], [-np.inf], [0.0]])
    out, _ = R.recur_sequence(x, g, "log", np.array([1e30]))
    np.testing.assert_allclose(out[1:, 0], [2.0, 5.0])
