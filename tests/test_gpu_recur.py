"""GPU parity of the channel-wise gated recurrence (recur_forward,
recur_backward, recur_step) against the fp64 oracle, and of its run together with
the cross attention.

Each element of each output is held to the bound that its own roundings leave
(oracle/recur_oracle.py, recur_bounds).
"""
import numpy as np
import pytest

import oracle.cross_oracle as X
import oracle.recur_oracle as R
from vda_testutil import from_device

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def V():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2609_20744_amd import vda
    return vda


def _hold(got, want, bound, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, what
    err = np.abs(got - want)
    ok = err <= bound + 1e-30  # subnormal outputs are flushed
    assert ok.all(), (what, int((~ok).sum()), float(np.nanmax(err / (bound + 1e-30))), np.argwhere(~ok)[:4].tolist())


class Case:
    def __init__(self, lens, C=64, gate="log", dtype="bf16", reverse=False, state=True, packed=None, lead=0, tail=0, fused=False,
                 slow=False, resets=False, seed=0):
        import torch
        rng = np.random.default_rng(seed + 17 * sum(lens) + C)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.gt = torch.float32 if gate == "log" else self.dt
        self.half, self.gate, self.reverse, self.lens, self.n, self.C = HALF[dtype], gate, reverse, lens, len(lens), C
        self.half_g = HALF["f32"] if gate == "log" else self.half
        self.packed = len(set(lens)) > 1 or lead > 0 or tail > 0 if packed is None else packed
        self.cu = lead + np.concatenate([[0], np.cumsum(lens)])
        T = int(self.cu[-1]) + tail

        def values(x, dt):
            t = torch.from_numpy(x).to(dt)
            return t, t.double().numpy()

        x, self.x = values(rng.standard_normal((T, C)), self.dt)
        z = rng.standard_normal((T, C)) + (9.0 if slow else 2.0)
        if gate == "log":
            z = -np.log1p(np.exp(-z))
            if resets:
                z[rng.random(T) < 0.05] = -np.inf
        g, self.g = values(z, self.gt)
        do, self.do = values(rng.standard_normal((T, C)), self.dt)
        lead_shape = (T,) if self.packed else (self.n, T // self.n)

        def place(t, dt):
            t = t.reshape(lead_shape + (C,))
            if not fused:
                return t.cuda()
            wide = torch.full(lead_shape + (3 * C,), 7.0, dtype=dt)
            wide[..., C:2 * C] = t
            return wide.cuda()[..., C:2 * C]

        self.dev = dict(x=place(x, self.dt), g=place(g, self.gt), dout=do.reshape(lead_shape + (C,)).cuda())
        self.S = self.dS = None
        self.S64, self.dS64 = np.zeros((self.n, C)), np.zeros((self.n, C))
        if state:
            self.S64, self.dS64 = (rng.standard_normal((self.n, C)).astype(np.float32).astype(np.float64) for _ in range(2))
            self.S, self.dS = (torch.from_numpy(s).float().cuda() for s in (self.S64, self.dS64))

    def options(self):
        import torch
        o = dict(gate=self.gate, reverse=self.reverse, state=self.S)
        if self.packed:
            o["cu_seqlens"] = torch.tensor(self.cu, dtype=torch.int32, device="cuda")
        return o

    def check(self, out=None, last=None, grads=None):
        for i in range(self.n):
            r = slice(self.cu[i], self.cu[i + 1])
            a = (self.x[r], self.g[r], self.gate, self.S64[i])
            if out is not None:
                want, bound = R.recur_sequence(*a, self.reverse), R.recur_bounds(*a, self.half, self.reverse)
                _hold(from_device(out.contiguous()).reshape(-1, self.C)[r], want[0], bound[0], ("out", i))
                _hold(from_device(last)[i], want[1], bound[1], ("state", i))
            if grads is not None:
                want = R.recur_sequence_backward(self.do[r], self.dS64[i], *a, self.reverse)
                bound = R.recur_bounds(*a, max(self.half, self.half_g), self.reverse, self.do[r], self.dS64[i])
                if self.half_g < self.half:  # an fp32 gate's gradient is rounded to fp32
                    tight = R.recur_bounds(*a, self.half_g, self.reverse, self.do[r], self.dS64[i])
                    bound = (bound[0], tight[1], bound[2])
                for t, w, b, name in zip(grads, want, bound, ("dx", "dg", "dstate")):
                    if t is not None:
                        got = from_device(t.contiguous())
                        got = got[i] if name == "dstate" else got.reshape(-1, self.C)[r]
                        _hold(got, w, b, (name, i))


CASES = {
    "one": dict(lens=[1], C=8),
    "eight": dict(lens=[8, 8], C=8),
    "nine": dict(lens=[9], C=136),
    "tile": dict(lens=[128, 128, 128], C=128),
    "tile_and_one": dict(lens=[129], C=72),
    "tiles": dict(lens=[515, 515], C=200),
    "long": dict(lens=[5003], C=40),
    "long_slow": dict(lens=[9000], C=16, slow=True),
    "packed": dict(lens=[70, 0, 1, 300, 33, 128, 0], C=64, lead=3, tail=5),
    "packed_long": dict(lens=[1, 2600, 0, 127, 900], C=24, lead=200, tail=1),
    "packed_many": dict(lens=[(7 * i) % 23 for i in range(150)], C=16),
    "packed_short": dict(lens=[40, 0, 60], C=16),
    "fused": dict(lens=[50, 50], C=64, fused=True),
    "fused_packed": dict(lens=[50, 700], C=64, fused=True, lead=2),
    "no_state": dict(lens=[260, 30], C=32, state=False),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reverse", [False, True], ids=["", "reverse"])
@pytest.mark.parametrize("gate", ["log", "logit", "norm"])
@pytest.mark.parametrize("name", CASES)
def test_forward_and_gradients(V, name, gate, reverse, dtype):
    print(name, gate, reverse, dtype, flush=True)
    c = Case(gate=gate, reverse=reverse, dtype=dtype, **CASES[name])
    out, last = V.recur_forward(c.dev["x"], c.dev["g"], return_state=True, **c.options())
    c.check(out, last.reshape(c.n, c.C))
    grads = V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, **c.options())
    assert (grads[2] is None) == (c.S is None)
    c.check(grads=grads)


def test_resets(V):
    """A log decay of -inf forgets the state, whatever it held, and has no gradient."""
    import torch
    for dtype in ("bf16", "f32"):
        c = Case([700, 40], C=16, resets=True, dtype=dtype)
        out, last = V.recur_forward(c.dev["x"], c.dev["g"], return_state=True, **c.options())
        c.check(out, last)
        grads = V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, **c.options())
        assert (grads[1][torch.isneginf(c.dev["g"])] == 0).all()
        with np.errstate(invalid="ignore"):
            c.check(grads=grads)


def test_saturated_gates(V):
    """Logits far out: a of 0 and of 1, finite everywhere."""
    import torch
    for gate in ("logit", "norm"):
        x = torch.randn(300, 16, device="cuda")
        g = torch.where(torch.rand(300, 16, device="cuda") < 0.5, 1.0, -1.0) * torch.tensor([30.0, 90.0, 1e4, 3e38], device="cuda").repeat(4)
        out = V.recur_forward(x, g, gate=gate)
        dx, dg, _ = V.recur_backward(torch.ones_like(x), x, g, gate=gate)
        want, _ = R.recur_sequence(from_device(x), from_device(g), gate, np.zeros(16))
        assert torch.isfinite(out).all() and torch.isfinite(dx).all() and torch.isfinite(dg).all()
        np.testing.assert_allclose(from_device(out), want, atol=300 * 2.0 ** -22)


def test_rows_outside_sequences_are_left(V):
    import torch
    c = Case([5, 400], C=16, gate="logit", lead=4, tail=6)
    out = torch.full_like(c.dev["x"], 3.0)
    _, last = V.recur_forward(c.dev["x"], c.dev["g"], out=out, return_state=True, **c.options())
    outs = (torch.full_like(out, 3.0), torch.full_like(out, 3.0), torch.zeros(2, 16, device="cuda"))
    V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, outs=outs, **c.options())
    c.check(out, last, outs)
    for t in (out, outs[0], outs[1]):
        assert (t[:4] == 3.0).all() and (t[-6:] == 3.0).all()


def test_fused_gradients_leave_what_lies_between(V):
    import torch
    c = Case([300, 300], C=32, gate="norm")
    wide = torch.full((2, 300, 96), 3.0, dtype=c.dt, device="cuda")
    outs = (wide[..., 32:64], wide[..., :32], torch.zeros(2, 32, device="cuda"))
    V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, outs=outs, **c.options())
    c.check(grads=outs)
    assert (wide[..., 64:] == 3.0).all()


def test_nan_stays_in_its_channel(V):
    import torch
    c = Case([300, 200], C=16)
    x = c.dev["x"].clone()
    x[310, 3] = float("nan")
    out, last = V.recur_forward(x, c.dev["g"], return_state=True, **c.options())
    ref, ref_last = V.recur_forward(c.dev["x"], c.dev["g"], return_state=True, **c.options())
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[300:, 3] = False
    assert torch.equal(out[keep], ref[keep]) and torch.equal(last[0], ref_last[0]) and torch.isnan(last[1, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["log", "logit", "norm"])
@pytest.mark.parametrize("n,t,m,C", [(1, 1, 1, 8), (5, 3, 9, 136), (200, 1, 201, 32)])
def test_step(V, n, t, m, C, gate, dtype):
    import torch
    rng = np.random.default_rng(n + C)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy(rng.standard_normal((n, t, C))).to(dt)
    g = torch.from_numpy(-np.abs(rng.standard_normal((n, t, C)))).to(torch.float32 if gate == "log" else dt)
    state = torch.from_numpy(rng.standard_normal((m, C))).float()
    slots = rng.permutation(m)[:n].astype(np.int32)
    if n > 1:
        slots[n // 2], slots[0] = -1, m
    pool, out = state.cuda(), torch.full((n, t, C), 9.0, dtype=dt, device="cuda")
    V.recur_step(x.cuda(), g.cuda(), pool, gate=gate, slots=torch.from_numpy(slots).cuda(), out=out)
    got, after = from_device(out), from_device(pool)
    touched = set()
    for i, s in enumerate(slots):
        if s < 0 or s >= m:
            assert (got[i] == 9.0).all()
            continue
        touched.add(int(s))
        a = (x[i].double().numpy(), g[i].double().numpy(), gate, state[s].double().numpy())
        (want, last), (b, bl) = R.recur_sequence(*a), R.recur_bounds(*a, HALF[dtype])
        _hold(got[i], want, b, i)
        _hold(after[s], last, bl, i)
    for s in set(range(m)) - touched:
        assert (after[s] == state[s].double().numpy()).all()


def test_same_bits_again(V):
    import torch
    c = Case([700, 0, 1, 2000], C=72, gate="norm")
    first = None
    for _ in range(4):
        got = [*V.recur_forward(c.dev["x"], c.dev["g"], return_state=True, **c.options()),
               *V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, **c.options())]
        got = [t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).clone() for t in got]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_garbage_in_work(V):
    import torch
    c = Case([700, 90, 2000], C=24, gate="logit")
    for backward in (False, True):
        n = V.recur_workspace(c.dev["x"], c.dev["g"], gate="logit", cu_seqlens=c.options()["cu_seqlens"], backward=backward)
        assert n > 0
        work = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        if backward:
            c.check(grads=V.recur_backward(c.dev["dout"], c.dev["x"], c.dev["g"], dstate=c.dS, work=work, **c.options()))
        else:
            c.check(*V.recur_forward(c.dev["x"], c.dev["g"], return_state=True, work=work, **c.options()))
        with pytest.raises(ValueError):
            V.recur_forward(c.dev["x"], c.dev["g"], work=work[:16], **c.options())


def test_offsets_out_of_order(V):
    """Values are undefined, what is around the tensors is not touched."""
    import torch
    guard, T, C = 512, 600, 16
    for cu in ([0, 600, 30, 600], [-5, 400, 10000, 20000], [600, 400, 200, 0], [7, 3, -9, 1 << 30], [0, 0, 0, 0]):
        x, g, do = (torch.randn(T, C, device="cuda").bfloat16() for _ in range(3))
        o = dict(gate="logit", cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        wides = [torch.full((T + 2 * guard, C), 5.0, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
        outs = [w[guard:guard + T] for w in wides]
        V.recur_forward(x, g, out=outs[0], **o)
        V.recur_backward(do, x, g, outs=(outs[1], outs[2], None), **o)
        torch.cuda.synchronize()
        for w in wides:
            assert (w[:guard] == 5.0).all() and (w[-guard:] == 5.0).all()


def test_rows_past_32_bits_of_offsets(V):
    """Rows of a fused projection, 2.1 GB and more from the tensor's begin."""
    import torch
    T, C, wide = 300000, 8, 8192
    fused = torch.zeros(T, wide, dtype=torch.bfloat16, device="cuda")
    x, g = fused[:, 8:16], fused[:, 16:24]
    x[-40:].normal_(), g[-40:].normal_()
    out, last = V.recur_forward(x, g, gate="logit", return_state=True)
    a = (from_device(x[-40:].contiguous()), from_device(g[-40:].contiguous()), "logit", np.zeros(C))
    _hold(from_device(out[-40:]), R.recur_sequence(*a)[0], R.recur_bounds(*a, 2.0 ** -8)[0], "out")
    _hold(from_device(last)[0] if last.dim() == 2 else from_device(last), R.recur_sequence(*a)[1], R.recur_bounds(*a, 0.0)[1], "state")


def test_captured_and_replayed(V):
    import torch
    c, e = (Case([700, 40], C=16, gate="norm", seed=s) for s in (0, 5))
    buf = {k: t.clone() for k, t in c.dev.items()}
    S, dS, o = c.S.clone(), c.dS.clone(), c.options()
    o["state"] = S
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def run():
        out, last = V.recur_forward(buf["x"], buf["g"], return_state=True, **o)
        return out, last, V.recur_backward(buf["dout"], buf["x"], buf["g"], dstate=dS, **o)

    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out, last, grads = run()
    for case in (c, e, c, e):
        for k, t in case.dev.items():
            buf[k].copy_(t)
        S.copy_(case.S), dS.copy_(case.dS)
        graph.replay()
        torch.cuda.synchronize()
        case.check(out, last, grads)
        run()
        torch.cuda.synchronize()


def test_refusals_of_the_binding(V):
    import torch
    x = torch.zeros(2, 6, 16, device="cuda", dtype=torch.bfloat16)
    f = x.float()
    for a, kw in (((x, x), dict(gate="log")), ((x, f), dict(gate="logit")), ((x, x), dict(gate="sigmoid")),
                  ((x[..., :12], f[..., :12]), {}), ((x[..., :12].contiguous(), f[..., :12].contiguous()), {}), ((x, f[:1]), {}),
                  ((x, f), dict(cu_seqlens=torch.zeros(3, dtype=torch.int32, device="cuda"))),
                  ((x, f), dict(state=torch.zeros(2, 8, device="cuda"))), ((x, f), dict(out=torch.zeros_like(f))),
                  ((x[:, :0], f[:, :0]), {}), ((x.transpose(0, 1), f.transpose(0, 1)), {}), ((x[0, 0], f[0, 0]), {})):
        with pytest.raises((ValueError, TypeError)):
            V.recur_forward(*a, **kw)
    with pytest.raises(ValueError):
        V.recur_backward(x[:1], x, f)
    with pytest.raises(ValueError):
        V.recur_backward(x.clone(), x, f, outs=(x.clone(), f.clone()))
    with pytest.raises(ValueError):
        V.recur_step(x, f, torch.zeros(1, 16, device="cuda"))
    with pytest.raises(ValueError):
        V.recur_step(x, f, torch.zeros(2, 8, device="cuda"))


def test_a_block_of_both(V):
    """A stream's block as it is used: the recurrence mixes the tokens, its output asks the prompt, and the
    gradients come back through both; then the same tokens one at a time, from the cached prompt and the state."""
    import torch
    B, L, S, H, d = 2, 70, 45, 4, 32
    C = H * d
    rng = np.random.default_rng(3)
    x, g, do = (torch.from_numpy(rng.standard_normal((B, L, C))).float() for _ in range(3))
    k, v = (torch.from_numpy(rng.standard_normal((B, S, H, d))).float() for _ in range(2))
    lens = [45, 20]
    h, _ = V.recur_forward(x.cuda(), g.cuda(), gate="norm", return_state=True)
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = h.reshape(B, L, H, d)
    y, lse = V.cross_forward(q, k.cuda(), v.cuda(), layout="tokens", k_lens=kl, return_lse=True)
    dq, dk, dv = V.cross_backward(do.reshape(B, L, H, d).cuda(), q, k.cuda(), v.cuda(), y, lse, layout="tokens", k_lens=kl)
    dx, dg, _ = V.recur_backward(dq.reshape(B, L, C), x.cuda(), g.cuda(), gate="norm")
    state, steps = torch.zeros(B, C, device="cuda"), []
    for t in range(L):
        ht = V.recur_step(x[:, t:t + 1].contiguous().cuda(), g[:, t:t + 1].contiguous().cuda(), state, gate="norm")
        steps.append(V.cross_step(ht.reshape(B, 1, H, d), k.cuda(), v.cuda(), k_lens=kl))
    steps = from_device(torch.cat(steps, 1))
    for i in range(B):
        seen = np.arange(S) < lens[i]
        xi, gi = x[i].double().numpy(), g[i].double().numpy()
        hi, _ = R.recur_sequence(xi, gi, "norm", np.zeros(C))
        want = X.cross_sequence(hi.reshape(L, H, d), k[i].double().numpy(), v[i].double().numpy(), seen, d ** -0.5,
                                do[i].double().numpy().reshape(L, H, d))
        rx, rg, _ = R.recur_sequence_backward(want[2].reshape(L, C), np.zeros(C), xi, gi, "norm", np.zeros(C))
        # fp32 throughout: sums of at most 70 * 45 terms in each of two operators, of the largest value's size.
        tol = 2 * 70 * 45 * 2.0 ** -24
        for got, ref in ((from_device(y)[i], want[0]), (steps[i], want[0]), (from_device(dk)[i], want[3]),
                         (from_device(dv)[i], want[4]), (from_device(dx)[i], rx), (from_device(dg)[i], rg)):
            assert np.abs(got - ref).max() <= tol * np.abs(ref).max()
