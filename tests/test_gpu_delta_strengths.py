"""GPU tests of write strengths of zero and of small gradients in the token-wise
gated delta rule: against the fp64 oracle (tolerances as in test_gpu_delta.py)
and against the same call with scaled gradients."""
import numpy as np
import pytest

from test_gpu_delta import TOL_F32_OUT, TOL_OUT, Case, _err

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def V():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2609_20744_amd import vda
    return vda


SHAPES = [dict(lens=[100], Hk=1, dk=32, dv=32), dict(lens=[70, 0, 130], Hk=2, group=2, dk=64, dv=128, layout="tokens"),
          dict(lens=[64 * 18 + 5], Hk=1, dk=128, dv=128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["32", "packed", "cut"])
def test_tokens_of_no_strength_hold_anything_finite(V, shape, dtype):
    """Padding inside a sequence: strength 0, keys of 1e10 and values of 1e20 there.  Nothing of them reaches a state,
    another token's output or another token's gradient."""
    print(f"strength 0, keys of 1e10, values of 1e20: {shape} {dtype}", flush=True)
    c = Case(dtype=dtype, **shape)
    T = c.host["beta"].shape[1]
    pad = np.random.default_rng(11).random(T) < 0.2
    pad[-1] = True
    c.host["beta"][:, pad] = 0.0
    c.host["v"][:, pad] *= 1e20
    c.host["k"][:, pad] *= 1e10
    for x in ("beta", "v", "k"):
        c.dev[x] = c.to_layout(c.host[x])
    c.check_forward(*c.forward(V))
    got, want = c.backward(V), c.oracle_backward()
    for name, g, w in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want):
        g = c.back(g)
        tol = TOL_OUT[dtype] if name in ("dq", "dk", "dv") else TOL_F32_OUT[dtype]
        for part in (pad, ~pad):  # (the strengths' gradients there are of the values' size)
            e = _err(g[:, part], w[:, part])
            assert e <= tol, (name, e, tol)
    assert _err(got[5].double().cpu().numpy(), want[5]) <= TOL_F32_OUT[dtype]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["32", "packed", "cut"])
def test_gradients_are_linear_in_the_loss(V, shape, dtype):
    """Gradients of a loss times 2^-40 are the gradients times 2^-40, strengths of zero among them: a power of two
    changes no rounding.  Products below 2^-126 may be lost, absolutely: with inputs of at most 2^7 and sums of at
    most 2^13 terms that is 2^-106."""
    print(f"gradients times 2^-40: {shape} {dtype}", flush=True)
    c = Case(dtype=dtype, rough=True, **shape)
    assert (c.host["beta"] == 0).any()
    big = c.backward(V)
    small = c.dev["do"], c.states[1]
    c.dev["do"], c.states[1] = small[0] * 2.0 ** -40, small[1] * 2.0 ** -40
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dS"), c.backward(V), big):
        off = (a.double() - b.double() * 2.0 ** -40).abs().max().item()
        assert off <= 2.0 ** -106, (name, off)


def test_no_strength_at_all(V):
    """Strengths of zero alone, from no state: outputs, states and all gradients but the strengths' are exactly zero."""
    c = Case(lens=[150], Hk=2, dk=64, dv=64, state=False)
    c.host["beta"][:] = 0.0
    c.dev["beta"] = c.to_layout(c.host["beta"])
    out, S = c.forward(V)
    assert (out == 0).all() and (S == 0).all()
    dq, dk, dv, dg, dbeta, _ = c.backward(V)
    assert all((t == 0).all() for t in (dq, dk, dv, dg))
    want = c.oracle_backward()[4]
    assert np.linalg.norm(want) > 0 and _err(c.back(dbeta), want) <= TOL_F32_OUT["bf16"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["32", "packed", "cut"])
def test_strengths_up_to_two_and_below_zero(V, shape, dtype):
    """The whole range that is stable for keys of length 1, and some tokens that are unlearned.  Writes are up to twice
    the errors that the tolerances count roundings of, so twice those."""
    import torch
    print(f"strengths in [-0.25, 2]: {shape} {dtype}", flush=True)
    c = Case(dtype=dtype, **shape)
    rng = np.random.default_rng(12)
    b = c.host["beta"]
    b.uniform_(0, 2, generator=torch.Generator().manual_seed(5))
    b[:, rng.random(b.shape[1]) < 0.1] = -0.25
    c.dev["beta"] = c.to_layout(b)
    out, S = c.forward(V)
    ref, last = c.oracle()
    assert _err(c.back(out), ref) <= 2 * TOL_OUT[dtype]
    assert _err(S.double().cpu().numpy(), last) <= 2 * TOL_F32_OUT[dtype]
    for name, g, w in zip(("dq", "dk", "dv", "dg", "dbeta"), c.backward(V), c.oracle_backward()):
        e, tol = _err(c.back(g), w), 2 * (TOL_OUT[dtype] if name in ("dq", "dk", "dv") else TOL_F32_OUT[dtype])
        print(name, f"{e:.1e}", flush=True)
        assert e <= tol, (name, e, tol)
