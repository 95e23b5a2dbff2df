"""GPU parity of the token-wise gated delta rule row by row: the norms of
test_gpu_delta.py are of whole tensors, in which one wrong token of thousands
does not show; here every token of every head is held to the fp64 oracle by
itself, the gates' gradients by groups of 64 tokens of a head and the states one
by one.  The error of a row is relative to its own norm or to the rows' root
mean square, whichever is larger.

Tolerances, bf16 storage: a rounding to bf16 is off by at most 2^-8.  On the way
to dv there is one, the output's; to out four (output, scores, writes, the state
that is read), to dq and dk as many (output, scores, and the writes or the
gradients in them), which do not all err to one side; 2^-12 stands for the values
held as two bf16 parts.  The kernels' roundings put into the chunk-wise form in
64 bits, on these cases with three seeds, gave at most 0.6 (dv), 2.1 (out), 3.0
(dq) and 1.5 (dk) times 2^-8, for states 4.4e-6, for the gates' gradients 4.6e-5.
fp32 storage: as in test_gpu_delta.py.
"""
import numpy as np
import pytest

from test_gpu_delta import CASES, IDS, TOL_F32_OUT, TOL_OUT, Case

TOL = {"bf16": dict(out=3 * 2.0 ** -8, dq=4 * 2.0 ** -8, dk=3 * 2.0 ** -8, dv=2.0 ** -8 + 2.0 ** -12, gates=TOL_F32_OUT["bf16"],
                    state=2 * 2.0 ** -16),
       "f32": dict.fromkeys(("out", "dq", "dk", "dv", "gates", "state"), TOL_OUT["f32"])}


@pytest.fixture(scope="module")
def V():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2609_20744_amd import vda
    return vda


def _worst(err, size):
    """Largest error of a row, relative to it or to the rows' root mean square."""
    if not size.size:
        return 0.0
    floor = np.sqrt(np.mean(size ** 2))
    assert np.isfinite(err).all()
    return float(np.max(err / np.maximum(size, floor if floor else 1.0)))


def rows_off(got, ref):
    return _worst(np.linalg.norm(got - ref, axis=-1), np.linalg.norm(ref, axis=-1))


def states_off(got, ref):
    return rows_off(got.reshape(*got.shape[:2], -1), ref.reshape(*ref.shape[:2], -1))


def gates_off(got, ref, cu):
    """[heads, tokens], by groups of up to 64 tokens of a sequence, of their root mean squares."""
    err, size = [], []
    for a, b in zip(cu[:-1], cu[1:]):
        for t in range(a, b, 64):
            s = slice(t, min(t + 64, b))
            err.append(np.sqrt(np.mean((got[:, s] - ref[:, s]) ** 2, axis=1)))
            size.append(np.sqrt(np.mean(ref[:, s] ** 2, axis=1)))
    return _worst(np.array(err), np.array(size))


def check(V, c):
    tol, real = TOL[c.dtype], slice(c.cu[0], c.cu[-1])
    out, S = c.forward(V)
    ref, last = c.oracle()
    off = {"out": rows_off(c.back(out)[:, real], ref[:, real]), "state": states_off(S.double().cpu().numpy(), last)}
    grads, want = c.backward(V), c.oracle_backward()
    for name, g, w in zip(("dq", "dk", "dv"), grads, want):
        off[name] = rows_off(c.back(g)[:, real], w[:, real])
    for name, g, w in zip(("dg", "dbeta"), grads[3:5], want[3:5]):
        off[name] = gates_off(c.back(g), w, c.cu)
    if grads[5] is not None:
        off["dS"] = states_off(grads[5].double().cpu().numpy(), want[5])
    print(c.dtype, {n: f"{e:.1e}" for n, e in off.items()}, flush=True)
    kind = {"dg": "gates", "dbeta": "gates", "dS": "state"}
    for name, e in off.items():
        assert e <= tol[kind.get(name, name)], (name, e, tol[kind.get(name, name)])


def _many(n, most, long_at, long):
    lens = [int(x) for x in np.random.default_rng(n).integers(0, most, n)]
    lens[long_at] = long
    return lens


TABLES = [dict(lens=_many(40, 40, 17, 64 * 40 + 3), Hk=4, group=2, dk=32, dv=32, layout="tokens", rough=True),
          dict(lens=_many(1024, 4, 1004, 64 * 17), Hk=1, dk=32, dv=32, layout="tokens"),
          dict(lens=_many(2050, 4, 2030, 64 * 17), Hk=1, dk=32, dv=32),
          dict(lens=[64 * 8, 64 * 9 + 5, 64 * 3, 1], Hk=2, dk=64, dv=64, rough=True),
          dict(lens=[64 * 9 - 1] * 3, Hk=2, dk=64, dv=64, uniform=True, rough=True),
          dict(lens=[64 * 6, 64 * 7], Hk=2, dk=64, dv=64, rough=True)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES + TABLES, ids=IDS + ["one_long", "1024", "2050", "8_to_9", "9_less_a_token", "6_and_7"])
def test_every_row(V, case, dtype):
    print(f"delta rows {str(case)[:100]} {dtype}", flush=True)
    check(V, Case(dtype=dtype, **case))


def test_one_wrong_row_is_seen():
    """One token of thousands, one state of hundreds, one gate of a group: each is past every tolerance."""
    rng = np.random.default_rng(0)
    most = max(TOL["bf16"].values())
    x = rng.standard_normal((4, 5000, 32))
    for change in (0.0, x[1, 4000]):  # lost, or another token's
        y = x.copy()
        y[2, 1234] = change
        assert rows_off(x, x) == 0 and rows_off(y, x) > 10 * most
    S = rng.standard_normal((300, 4, 16, 16))
    y = S.copy()
    y[17, 2] = y[18, 2]
    assert states_off(y, S) > 10 * most
    g = rng.standard_normal((4, 5000))
    y = g.copy()
    y[3, 70] = -y[3, 70]
    assert gates_off(g, g, [0, 40, 5000]) == 0 and gates_off(y, g, [0, 40, 5000]) > most
