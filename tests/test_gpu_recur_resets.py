"""A log decay of -inf resets the recurrence's state whatever it held, infinities and NaN
of a slot that was used before (or never filled) included."""
import numpy as np
import pytest

from test_gpu_recur import Case, V  # noqa: F401  (V: the fixture)

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), float("-inf")]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reverse", [False, True], ids=["", "reverse"])
@pytest.mark.parametrize("lens,at", [([1], 0), ([40], 0), ([40], 17), ([300], 3), ([300], 131), ([5000], 0), ([5000], 2500),
                                     ([700, 0, 90, 2600], 40)], ids=str)
def test_a_reset_forgets_any_state(V, lens, at, reverse, dtype, bad):
    """The state that sequences start from is `bad` in every other channel; their token `at`, in the order of the recurrence,
    resets.  From there on outputs, and everywhere the gradients that do not meet that state, are those of a start from 0."""
    import torch
    c = Case(lens, C=24, reverse=reverse, dtype=dtype, packed=True)
    x, g = c.dev["x"], c.dev["g"].clone()
    rows, since = [], torch.zeros(len(x), dtype=torch.bool, device="cuda")
    for a, b in zip(c.cu[:-1], c.cu[1:]):
        if b > a:
            t = b - 1 - at if reverse else a + at
            rows.append(int(t))
            since[a:t + 1] = reverse
            since[t:b] |= not reverse
    g[rows] = -np.inf
    o = c.options()
    zero = torch.zeros_like(c.S)
    start = zero.clone()
    start[:, ::2] = bad
    want, want_last = V.recur_forward(x, g, return_state=True, **{**o, "state": zero})
    out, last = V.recur_forward(x, g, return_state=True, **{**o, "state": start})
    full = torch.tensor([n > 0 for n in lens], device="cuda")
    assert torch.equal(out[since], want[since]) and torch.equal(last[full], want_last[full])
    assert torch.isfinite(want[since]).all()
    wx, wg, ws = V.recur_backward(c.dev["dout"], x, g, dstate=c.dS, **{**o, "state": zero})
    dx, dg, ds = V.recur_backward(c.dev["dout"], x, g, dstate=c.dS, **{**o, "state": start})
    assert torch.equal(dx, wx) and torch.equal(ds, ws) and torch.equal(dg[since], wg[since])
    assert (dg[rows] == 0).all()


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_resets_a_slot(V, dtype, bad):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    state = torch.full((4, 16), bad, device="cuda")
    x = torch.randn(2, 3, 16, device="cuda").to(dt)
    g = -torch.rand(2, 3, 16, device="cuda")
    g[:, 1] = -np.inf
    out = V.recur_step(x, g, state, slots=torch.tensor([3, 1], dtype=torch.int32, device="cuda"))
    assert not torch.isfinite(out[:, 0]).any() and torch.equal(out[:, 1], x[:, 1])
    h = torch.addcmul(x[:, 2].float(), g[:, 2].exp(), x[:, 1].float())
    # A product, a sum, an exponential and its argument, and the output are rounded.
    tol = 6 * 2.0 ** -24 * (x[:, 1].float().abs() + x[:, 2].float().abs())
    assert ((state[[3, 1]] - h).abs() <= tol).all()
    assert ((out[:, 2].float() - h).abs() <= tol + torch.finfo(dt).eps / 2 * h.abs()).all()
    assert not torch.isfinite(state[[0, 2]]).any()
