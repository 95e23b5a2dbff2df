"""The cross attention's gradients where a mask or length hides states: what dout and
q hold does not reach hidden states, and D is summed over the states that are seen,
wherever they stand."""
import numpy as np
import pytest

import oracle.cross_oracle as X
from test_gpu_cross import Case, V  # noqa: F401  (V: the fixture)
from vda_testutil import from_device

pytestmark = pytest.mark.gpu


def _run(V, c):
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    return out, lse, V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)


HIDDEN = {
    "nothing_seen": dict(lq=[140, 40], lk=[90, 70], Hq=2, Hk=1, mask="first"),
    "padded": dict(lq=[70, 70], lk=[200, 200], Hq=2, Hk=2, lens=[0, 130]),
    "holes_in_tiles": dict(lq=[70], lk=[300], Hq=4, Hk=2, d=128, mask="holes"),
    "ranges": dict(lq=[3000], lk=[150], Hq=1, Hk=1, d=32, mask="holes"),
}


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["dout", "q"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", HIDDEN)
def test_hidden_states_have_no_gradient(V, name, dtype, where, bad):
    """A NaN or infinity of a query or of its output's gradient: gradients of what it meets are undefined, those of states that
    nothing sees are 0, and a query that sees nothing has none."""
    import torch
    c = Case(dtype=dtype, **HIDDEN[name])
    d, o = c.dev, c.options()
    x = d[where].view(-1, c.Hq, c.d)
    x[3] = bad  # a token of the first sequence, all heads
    out, lse, (dq, dk, dv) = _run(V, c)
    hidden = torch.from_numpy(~c.seen).cuda()
    assert bool(hidden.any())
    for g in (dk, dv):
        assert (g.view(-1, c.Hk, c.d)[hidden] == 0).all()
    if not c.seen[:c.ck[1]].any():
        assert (dq.view(-1, c.Hq, c.d)[:c.cq[1]] == 0).all()
    # Another sequence's gradients are as ever.
    for i in range(1, c.n):
        r, s = slice(c.cq[i], c.cq[i + 1]), slice(c.ck[i], c.ck[i + 1])
        a = (c.q[r], c.k[s], c.v[s], c.seen[s], c.scale)
        want, bound = X.cross_sequence(*a, c.do[r]), X.cross_bounds(*a, c.half, c.do[r])
        for got, w, b in zip((dq.view(-1, c.Hq, c.d)[r], dk.view(-1, c.Hk, c.d)[s], dv.view(-1, c.Hk, c.d)[s]), want[2:], bound[2:]):
            assert (np.abs(from_device(got.contiguous()) - w) <= b + 1e-30).all()
