"""Pins of oracle/delta_oracle.py: closed forms of the token-wise rule, its
relation to the frame-wise operator, and its gradients and the rotation's by
differences."""
import numpy as np
import pytest

import oracle.delta_oracle as D
import oracle.vda_oracle as O


def _problem(rng, Hk=2, group=2, T=7, dk=5, dv=4, n=2):
    Hv = Hk * group
    q, k = rng.standard_normal((2, Hk, T, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    v = rng.standard_normal((Hv, T, dv))
    g, beta = -rng.random((Hv, T)), rng.random((Hv, T))
    return q, k, v, g, beta, rng.standard_normal((n, Hv, dv, dk))


def test_single_token_closed_form():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((3, 6))
    k /= np.linalg.norm(k)
    S0 = rng.standard_normal((6, 6))
    o, S = D.delta_head(q[None], k[None], v[None], np.array([-0.3]), np.array([1.0]), S0, 0.5)
    # beta = 1 and |k| = 1: the new state answers k with v exactly.
    assert np.allclose(S @ k, v, atol=1e-13)
    # ... and keeps (decayed) what is orthogonal to k.
    u = q - (q @ k) * k
    assert np.allclose(S @ u, np.exp(-0.3) * (S0 @ u), atol=1e-13)
    assert np.allclose(o[0], 0.5 * (S @ q), atol=1e-14)


def test_frames_of_one_token_are_the_rule():
    """A frame of one token of the joint solve (Eq. 5) is the token rule with
    beta' = beta / (1 + beta |k|^2) (Sherman-Morrison), no decay."""
    rng = np.random.default_rng(2)
    F, dk, dv = 6, 5, 4
    k, v, beta = rng.standard_normal((F, dk)), rng.standard_normal((F, dv)), rng.random(F)
    S = O.text_state(k[None, :1], v[None, :1], beta[None, :1])[0]
    _, mine = D.delta_head(k[:1], k[:1], v[:1], np.zeros(1), beta[:1] / (1 + beta[:1] * (k[:1] ** 2).sum(-1)),
                           np.zeros((dv, dk)), 1.0)
    assert np.allclose(S, mine, atol=1e-13)


def test_reset_forgets_everything_before():
    rng = np.random.default_rng(3)
    q, k, v, g, beta, S = _problem(rng, Hk=1, group=1, n=1)
    g[0, 3] = -np.inf
    o, _ = D.delta_sequences(q, k, v, g, beta, [0, 7], S, 1.0)
    o2, _ = D.delta_sequences(q[:, 3:], k[:, 3:], v[:, 3:], np.where(np.arange(4) == 0, 0.0, g[:, 3:]), beta[:, 3:],
                              [0, 4], None, 1.0)
    assert np.allclose(o[:, 3:], o2, atol=1e-13)


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "S"])
def test_gradients_are_differences(name):
    rng = np.random.default_rng(4)
    q, k, v, g, beta, S = _problem(rng)
    cu = [0, 4, 7]
    do, dS = rng.standard_normal(v.shape), rng.standard_normal(S.shape)
    args = dict(q=q, k=k, v=v, g=g, beta=beta, S=S)

    def loss():
        o, last = D.delta_sequences(args["q"], args["k"], args["v"], args["g"], args["beta"], cu, args["S"], 0.7)
        return np.sum(o * do) + np.sum(last * dS)

    grads = dict(zip(("q", "k", "v", "g", "beta", "S"),
                     D.delta_sequences_backward(do, dS, q, k, v, g, beta, cu, S, 0.7)))
    for _ in range(12):
        u = rng.standard_normal(args[name].shape)
        x, h = args[name], 1e-6
        args[name] = x + h * u
        up = loss()
        args[name] = x - h * u
        down = loss()
        args[name] = x
        # Central differences: h^2 / 6 of the third derivative and 2^-52 / h of the loss.
        assert np.isclose((up - down) / (2 * h), np.sum(grads[name] * u), rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("l2", [True, False])
def test_rope_turns_and_its_gradient(interleaved, l2):
    rng = np.random.default_rng(5)
    x, dy = rng.standard_normal((2, 6, 12))
    axes, pos = (1, 2, 2), rng.integers(0, 50, (6, 3))
    f = rng.random(5).astype(np.float32)
    y = D.rope_head(x, pos, f, axes, interleaved, l2)
    # Lengths of the pairs are kept (of the normalised token with l2); the last two channels stay.
    want = x / np.sqrt((x * x).sum(-1, keepdims=True) + 1e-6) if l2 else x
    assert np.allclose((y * y).sum(-1), (want * want).sum(-1), atol=1e-13)
    assert np.allclose(y[:, 10:], want[:, 10:], atol=1e-15)
    # Two tokens' product depends on the difference of their positions only.
    if not l2:
        a = D.rope_head(x[:1], pos[:1] + 7, f, axes, interleaved, l2) @ D.rope_head(dy[:1], pos[1:2] + 7, f, axes, interleaved, l2).T
        b = D.rope_head(x[:1], pos[:1], f, axes, interleaved, l2) @ D.rope_head(dy[:1], pos[1:2], f, axes, interleaved, l2).T
        assert np.allclose(a, b, atol=1e-12)
    dx = D.rope_head_backward(dy, x, pos, f, axes, interleaved, l2)
    for _ in range(5):
        u, h = rng.standard_normal(x.shape), 1e-6
        d = (np.sum(D.rope_head(x + h * u, pos, f, axes, interleaved, l2) * dy)
             - np.sum(D.rope_head(x - h * u, pos, f, axes, interleaved, l2) * dy)) / (2 * h)
        assert np.isclose(d, np.sum(dx * u), rtol=1e-6, atol=1e-7)


def test_grid_positions():
    p = D.grid_positions(14, 2, 3, 5)
    assert p[0].tolist() == [5, 0, 0] and p[4].tolist() == [5, 1, 1] and p[13].tolist() == [7, 0, 1]
