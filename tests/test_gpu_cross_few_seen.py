"""The cross attention's gradients where a mask leaves few of many states: D is summed
from the weights of the states that are seen, as where there are no others."""
import numpy as np
import pytest

import oracle.cross_oracle as X
from test_gpu_cross import Case, V  # noqa: F401  (V: the fixture)

pytestmark = pytest.mark.gpu


def _see(c, at):
    """Only the states `at` are seen; the others hold NaN and infinities."""
    import torch
    c.seen[:] = False
    c.seen[at] = True
    c.mask = torch.from_numpy(c.seen.copy())
    hidden = torch.from_numpy(~c.seen).cuda()
    c.dev["k"].view(-1, c.Hk, c.d)[hidden], c.dev["v"].view(-1, c.Hk, c.d)[hidden] = float("nan"), float("inf")
    return c


def _run(V, c):
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    return out, lse, V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)


SHAPES = {
    "one_sequence": dict(lq=[300], lk=[600], Hq=4, Hk=2, d=128),
    "ranges": dict(lq=[40], lk=[5000], Hq=2, Hk=2, d=64),  # few rows: the states are shared out
    "equal": dict(lq=[70, 70], lk=[321, 321], Hq=2, Hk=1, d=32),
    "packed": dict(lq=[33, 0, 200, 5], lk=[900, 7, 257, 64], Hq=3, Hk=1, d=64),
    "many": dict(lq=[130] * 70, lk=[260] * 70, Hq=2, Hk=2, d=32),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("place", ["first", "inside", "last"])
@pytest.mark.parametrize("name", SHAPES)
def test_one_of_many_seen_has_no_gradient_of_scores(V, name, place, dtype):
    """A softmax over one state is constant, wherever that state stands: dq and dk are zeros."""
    c = Case(dtype=dtype, **SHAPES[name])
    at = {"first": c.ck[:-1], "inside": c.ck[:-1] + (np.diff(c.ck) * 2) // 3, "last": c.ck[1:] - 1}[place]
    out, lse, (dq, dk, dv) = _run(V, _see(c, at))
    c.check(out, lse, (dq, dk, dv))
    assert not dq.any() and not dk.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seen", [2, 255, 256, 257, 300])
@pytest.mark.parametrize("name", ["one_sequence", "ranges"])
def test_counts_about_the_limit(V, name, seen, dtype):
    c = Case(dtype=dtype, **SHAPES[name])
    at = np.sort(np.random.default_rng(seen).permutation(c.lk[0])[:seen])
    out, lse, grads = _run(V, _see(c, at))
    c.check(out, lse, grads)


@pytest.mark.parametrize("seen", [2, 5, 30])
@pytest.mark.parametrize("lk", [300, 600, 2000])
def test_gradients_of_few_seen_states_keep_their_norm(V, lk, seen):
    """What roundings leave of a gradient's norm.  One to bf16 is off by 2^-8 of a value's power of two at most, evenly, so by
    2^-8 / sqrt(3) of that in the root mean square, and that is 0.73 of the values' own: 0.0017 of a vector's norm.  dq and
    dk have two (score gradients, result), dv two (weights, result): 0.0017 sqrt(2) = 0.0024, and of a sum over thousands of
    values no more than a tenth beyond.  D taken from a rounded output would be a third, larger the fewer share the weight."""
    c = Case(lq=[130] * 4, lk=[lk] * 4, Hq=4, Hk=4, d=128, spread=1.5)
    rng = np.random.default_rng(seen)
    out, lse, grads = _run(V, _see(c, np.concatenate([a + rng.permutation(lk)[:seen] for a in c.ck[:-1]])))
    dq, dk, dv = (c.tokens(x, "tokens") for x in grads)
    off = np.zeros((3, 2))
    for i in range(c.n):
        r, s = slice(c.cq[i], c.cq[i + 1]), slice(c.ck[i], c.ck[i + 1])
        want = X.cross_sequence(c.q[r], c.k[s], c.v[s], c.seen[s], c.scale, c.do[r])[2:]
        for x, g, w in zip(off, (dq[r], dk[s], dv[s]), want):
            x += (np.sum((g - w) ** 2), np.sum(w ** 2))
    assert (np.sqrt(off[:, 0] / off[:, 1]) < 0.0026).all(), np.sqrt(off[:, 0] / off[:, 1])
