"""GPU parity of the token-wise gated delta rule (delta_forward,
delta_backward, delta_step) against the fp64 oracle.

Errors are 2-norms relative to the oracle's output.  A rounding to bf16 is off
by at most 2^-8 of the value, one to two bf16 parts by 2^-16, one to fp32 by
2^-24; the rule does not grow errors (|k| = 1, 0 <= beta <= 1, g <= 0), and
roundings of different values are as likely up as down, so the roundings on a
path are counted, worst case each:

* out, dq, dk, dv of bf16 storage: the output, the scores, the writes and the
  states that a product reads: 4 * 2^-8;
* states, dg, dbeta of bf16 storage: S, X, T and N as two parts, and their
  lo * lo products left out, twice in the backward pass and once more where
  they are kept: 10 * 2^-16;
* fp32 storage and the recurrent form: sums of up to 128 + 64 products, three in a row, 3 * 192 * 2^-24;
  the recurrent form in bf16 rounds its output only.
"""
import numpy as np
import pytest

import oracle.delta_oracle as D
from vda_testutil import from_device

pytestmark = pytest.mark.gpu

TOL_OUT = {"bf16": 4 * 2.0 ** -8, "f32": 3 * 192 * 2.0 ** -24}
TOL_F32_OUT = {"bf16": 10 * 2.0 ** -16, "f32": 3 * 192 * 2.0 ** -24}


@pytest.fixture(scope="module")
def V():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2609_20744_amd import vda
    return vda


def _err(got, ref):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert got.shape == ref.shape
    n = np.linalg.norm(ref)
    return np.linalg.norm(got - ref) / n if n else np.linalg.norm(got - ref)


class Case:
    """A problem in the heads layout on the host (the stored values, in 64 bits) and on the device in its layout."""

    def __init__(self, lens, Hk=2, group=1, dk=64, dv=64, dtype="bf16", layout="heads", state=True, rough=False,
                 uniform=False, lead=0, tail=0, seed=0):
        import torch
        rng = np.random.default_rng(seed + 1000 * sum(lens) + dk + dv)
        self.layout, self.dtype, self.uniform = layout, dtype, uniform
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        Hv, n = Hk * group, len(lens)
        self.cu = np.concatenate([[0], np.cumsum(lens)]) + lead
        T = int(self.cu[-1]) + tail

        def store(x):
            return torch.from_numpy(x).to(self.dt)

        def unit(*s):
            x = rng.standard_normal(s) + 0.7 * rng.standard_normal(s[-1])
            return store(x / np.linalg.norm(x, axis=-1, keepdims=True))

        q, k = unit(Hk, T, dk), unit(Hk, T, dk)
        v, do = store(rng.standard_normal((Hv, T, dv))), store(rng.standard_normal((Hv, T, dv)))
        g = -np.log1p(np.exp(2 * rng.standard_normal((Hv, T)) - 3))
        beta = 1 / (1 + np.exp(-1.5 * rng.standard_normal((Hv, T))))
        if rough:
            g[rng.random((Hv, T)) < 0.02] = -np.inf
            g[rng.random((Hv, T)) < 0.1] = 0.0
            beta[rng.random((Hv, T)) < 0.2] = 0.0
            beta[rng.random((Hv, T)) < 0.1] = 1.0
            kk = k.float().numpy()
            kk[:, 1::3] = kk[:, 0:-1:3][:, :kk[:, 1::3].shape[1]]  # repeated keys
            k = store(kk)
        g, beta = torch.from_numpy(g).float(), torch.from_numpy(beta).float()
        self.S = torch.from_numpy(0.3 * rng.standard_normal((n, Hv, dv, dk))).float() if state else None
        self.dS = torch.from_numpy(0.3 * rng.standard_normal((n, Hv, dv, dk))).float() if state else None
        self.scale = float(np.float32(dk ** -0.5))
        self.host = dict(q=q, k=k, v=v, g=g, beta=beta, do=do)
        self.dev = {x: self.to_layout(t) for x, t in self.host.items()}
        self.states = [None if s is None else s.cuda() for s in (self.S, self.dS)]
        self.cu_dev = None if uniform else torch.tensor(self.cu, dtype=torch.int32, device="cuda")
        self.kw = dict(cu_seqlens=self.cu_dev, layout=layout, scale=self.scale)

    def to_layout(self, t):
        n = len(self.cu) - 1
        if self.uniform:  # [H, n * L, ..] -> [n, H, L, ..]
            t = t.unflatten(1, (n, -1)).transpose(0, 1)
            return (t if self.layout == "heads" else t.transpose(1, 2)).contiguous().cuda()
        return (t if self.layout == "heads" else t.transpose(0, 1)).contiguous().cuda()

    def back(self, t):
        t = t.cpu()
        if self.layout == "tokens":
            t = t.transpose(1, 2) if self.uniform else t.transpose(0, 1)
        if self.uniform:
            t = t.transpose(0, 1).flatten(1, 2)
        return t.double().numpy()

    def ref(self, x):
        return self.host[x].double().numpy()

    def oracle(self):
        S = None if self.S is None else self.S.double().numpy()
        return D.delta_sequences(*(self.ref(x) for x in ("q", "k", "v", "g", "beta")), self.cu, S, self.scale)

    def oracle_backward(self):
        S, dS = (None if s is None else s.double().numpy() for s in (self.S, self.dS))
        return D.delta_sequences_backward(self.ref("do"), dS, *(self.ref(x) for x in ("q", "k", "v", "g", "beta")),
                                          self.cu, S, self.scale)

    def forward(self, V, **kw):
        d = self.dev
        return V.delta_forward(d["q"], d["k"], d["v"], d["g"], d["beta"], state=self.states[0], return_state=True,
                               **{**self.kw, **kw})

    def backward(self, V, **kw):
        d = self.dev
        return V.delta_backward(d["do"], d["q"], d["k"], d["v"], d["g"], d["beta"], state=self.states[0],
                                dstate=self.states[1], **{**self.kw, **kw})

    def check_forward(self, out, S):
        ref, last = self.oracle()
        real = slice(self.cu[0], self.cu[-1])
        assert _err(self.back(out)[:, real], ref[:, real]) <= TOL_OUT[self.dtype]
        assert _err(S.double().cpu().numpy(), last) <= TOL_F32_OUT[self.dtype]

    def check_backward(self, grads):
        ref = self.oracle_backward()
        real = slice(self.cu[0], self.cu[-1])
        for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta", "dS"), grads, ref):
            if got is None:
                continue
            tol = TOL_OUT[self.dtype] if name in ("dq", "dk", "dv") else TOL_F32_OUT[self.dtype]
            if name == "dS":
                e = _err(got.double().cpu().numpy(), want)
            else:
                e = _err(self.back(got)[:, real], want[:, real])
            assert e <= tol, (name, e, tol)


CASES = [
    dict(lens=[1], dk=32, dv=32),
    dict(lens=[1, 1, 1], uniform=True, layout="tokens"),
    dict(lens=[2], group=3),
    dict(lens=[63], dk=128, dv=128, state=False),
    dict(lens=[64], dk=128, dv=64, layout="tokens"),
    dict(lens=[65], dk=64, dv=128, rough=True),
    dict(lens=[129], dk=32, dv=128, group=2, rough=True),
    dict(lens=[77, 77, 77], uniform=True, dk=128, dv=128, group=2),
    dict(lens=[130, 130], uniform=True, layout="tokens", dk=128, dv=32, Hk=3, rough=True),
    dict(lens=[0, 1, 64, 65, 0, 200, 63, 0], layout="tokens", dk=64, dv=64, group=2, rough=True),
    dict(lens=[5, 0, 100], lead=3, tail=70, dk=128, dv=128),
    dict(lens=[0, 0], dk=32, dv=64, tail=2),
    # Long enough to be cut into segments: one sequence, and uneven ones.
    dict(lens=[64 * 18 + 7], Hk=1, group=2, dk=128, dv=128, rough=True),
    dict(lens=[64 * 21], Hk=1, dk=64, dv=32, state=False),
    dict(lens=[30, 64 * 17 + 1, 0, 300], Hk=1, dk=32, dv=64, layout="tokens"),
    dict(lens=[64 * 20 - 1] * 2, uniform=True, Hk=1, dk=128, dv=64, layout="tokens"),
]
IDS = ["_".join(str(x) for x in (c["lens"] if len(c["lens"]) < 4 else ["ragged"])) + f"_{c.get('dk', 64)}x{c.get('dv', 64)}"
       for c in CASES]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(V, case, dtype):
    print(f"delta forward {case} {dtype}", flush=True)
    c = Case(dtype=dtype, **case)
    c.check_forward(*c.forward(V))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(V, case, dtype):
    print(f"delta backward {case} {dtype}", flush=True)
    c = Case(dtype=dtype, **case)
    c.check_backward(c.backward(V))


@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_rows_outside_the_sequences_stay(V, layout):
    import torch
    c = Case(lens=[70, 0, 9], lead=5, tail=66, layout=layout, dk=32, dv=32)
    mark = lambda t: torch.full_like(t, 7.0)  # noqa: E731
    out = mark(c.dev["v"])
    c.forward(V, out=out)
    outs = [mark(c.dev[x]) for x in ("q", "k", "v", "g", "beta")] + [torch.empty_like(c.states[0])]
    c.backward(V, outs=outs)
    for t in [out] + outs[:5]:
        t = c.back(t)
        assert (t[:, :5] == 7).all() and (t[:, c.cu[-1]:] == 7).all()
        assert not (t[:, 5:c.cu[-1]] == 7).all()


def test_nan_stays_in_its_sequence_and_head(V):
    """NaN outside every sequence is not read; NaN in one sequence and head reaches no other."""
    import torch
    c = Case(lens=[70, 90, 40], lead=4, tail=30, Hk=2, group=1, dk=64, dv=64)
    clean, grads = c.forward(V), c.backward(V)
    for x in ("q", "k", "v", "g", "beta", "do"):
        c.dev[x][:, :4] = float("nan")
        c.dev[x][:, c.cu[-1]:] = float("inf")
    out, S = c.forward(V)
    assert torch.equal(out[:, 4:c.cu[-1]], clean[0][:, 4:c.cu[-1]]) and torch.equal(S, clean[1])
    for a, b in zip(c.backward(V)[:5], grads):
        assert torch.equal(a[:, 4:c.cu[-1]], b[:, 4:c.cu[-1]])
    c.dev["k"][1, c.cu[1] + 70] = float("nan")
    out, S = c.forward(V)
    assert torch.equal(out[0, 4:c.cu[-1]], clean[0][0, 4:c.cu[-1]])
    for s in (slice(4, c.cu[1]), slice(c.cu[2], c.cu[3]), slice(c.cu[1], c.cu[1] + 64)):
        assert torch.equal(out[1, s], clean[0][1, s])
    assert out[1, c.cu[1] + 70:c.cu[2]].isnan().any() and S[1, 1].isnan().any()
    assert torch.equal(S[0], clean[1][0]) and torch.equal(S[2], clean[1][2])


def test_resets_and_strong_decays(V):
    """Decays of exactly zero, by -inf and by far below fp32's range, and a chunk whose decays sum to thousands."""
    import torch
    c = Case(lens=[200], Hk=1, dk=64, dv=64)
    for t, g in ((0, -1e30), (30, -np.inf), (31, -300.0), (64, -np.inf), (100, -150.0), (101, -150.0)):
        c.host["g"][:, t] = g
    c.host["g"][:, 130:180] = -90.0
    c.dev["g"] = c.to_layout(c.host["g"])
    c.check_forward(*c.forward(V))
    grads = c.backward(V)
    c.check_backward(grads)
    assert float(grads[3][0, 30]) == 0.0 and float(grads[3][0, 64]) == 0.0 and torch.isfinite(grads[3]).all()


def test_zero_strength_writes_nothing(V):
    import torch
    c = Case(lens=[100], Hk=1, dk=32, dv=32)
    c.host["beta"][:] = 0.0
    c.host["beta"][:, 50] = -0.0
    c.dev["beta"] = c.to_layout(c.host["beta"])
    out, S = c.forward(V)
    c.check_forward(out, S)
    c.check_backward(c.backward(V))


def test_offsets_out_of_range_are_bounded(V):
    """Offsets below 0 or past T mean the nearest bound."""
    import torch
    c = Case(lens=[40, 100], Hk=2, dk=64, dv=64)
    want = c.forward(V)
    c.kw["cu_seqlens"] = torch.tensor([-5, 40, 100000], dtype=torch.int32, device="cuda")
    got = c.forward(V)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("lens,Hk", [([300, 70], 4), ([64 * 18], 1)])
def test_same_bits_again(V, lens, Hk):
    import torch
    c = Case(lens=lens, Hk=Hk, group=2, dk=128, dv=128, rough=True)
    a, b = c.forward(V), c.forward(V)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    a, b = c.backward(V), c.backward(V)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_dirty_workspace_does_not_matter(V):
    import torch
    c = Case(lens=[64 * 17 + 5, 100], Hk=1, group=2, dk=64, dv=64)
    want, grads = c.forward(V), c.backward(V)
    d = c.dev
    for backward in (False, True):
        n = V.delta_workspace(d["q"], d["k"], d["v"], d["g"], d["beta"], cu_seqlens=c.cu_dev, backward=backward)
        work = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")  # NaN in every type
        got = c.backward(V, work=work) if backward else c.forward(V, work=work)
        assert all(torch.equal(x, y) for x, y in zip(got, grads if backward else want))
    with pytest.raises(ValueError):
        c.forward(V, work=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_graphs_and_streams(V):
    """Two captured graphs (forward and backward, workspaces of their own) replayed in turn and side by side, with the
    program's eager calls between; and a call on another stream than the current one."""
    import torch
    c = Case(lens=[64 * 17, 90], Hk=1, group=2, dk=64, dv=64, rough=True)
    want, grads = c.forward(V), c.backward(V)
    torch.cuda.synchronize()
    gf, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(gf):
        captured = c.forward(V)
    with torch.cuda.graph(gb):
        captured_grads = c.backward(V)
    side = torch.cuda.Stream()
    for turn in range(4):
        for t in list(captured) + list(captured_grads):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        gf.replay()
        eager = c.forward(V)
        with torch.cuda.stream(side):
            gb.replay()
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, want)), turn
        assert all(torch.equal(x, y) for x, y in zip(eager, want)), turn
        assert all(torch.equal(x, y) for x, y in zip(captured_grads, grads)), turn
    got = c.forward(V, stream=side)
    got2 = c.backward(V, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(torch.equal(x, y) for x, y in zip(got2, grads))


def test_argument_errors(V):
    import torch
    c = Case(lens=[20], Hk=2, group=2, dk=32, dv=32)
    d = c.dev
    args = [d[x] for x in ("q", "k", "v", "g", "beta")]
    for i, bad in [(1, d["k"][:, :10].contiguous()), (2, d["v"][:3].contiguous()), (3, d["g"].double()),
                   (4, d["beta"][:, :10].contiguous()), (0, d["q"].float()), (2, d["v"].transpose(1, 2)),
                   (1, d["k"].cpu())]:
        with pytest.raises(ValueError):
            V.delta_forward(*args[:i], bad, *args[i + 1:], **c.kw)
    for kw in (dict(layout="rows"), dict(cu_seqlens=c.cu_dev.long()), dict(state=torch.zeros(1, 4, 32, 31, device="cuda")),
               dict(out=d["q"])):
        with pytest.raises(ValueError):
            V.delta_forward(*args, **{**c.kw, **kw})
    with pytest.raises(ValueError):  # not in place
        c.forward(V, state_out=c.states[0])
    with pytest.raises(ValueError):
        V.delta_backward(d["do"][:, :5].contiguous(), *args, **c.kw)


# ---------------------------------------------------------------------------------------------------------------------
# Tables of many and uneven sequences; large tensors
# ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_long_sequence_among_many(V, dtype):
    """Sequences and heads that fill the device by themselves: the long one alone is cut into segments."""
    lens = [int(x) for x in np.random.default_rng(3).integers(0, 40, 40)]
    lens[17] = 64 * 40 + 3
    c = Case(lens, Hk=4, group=2, dk=32, dv=32, dtype=dtype, layout="tokens", rough=True)
    c.check_forward(*c.forward(V))
    c.check_backward(c.backward(V))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,uniform", [([64 * 8], False), ([64 * 8 + 1], False), ([64 * 9], True),
                                          ([64 * 8, 64 * 9 + 5, 64 * 3, 1], False), ([64 * 9 - 1] * 3, True),
                                          ([64 * 6], True), ([64 * 6 + 1], True), ([64 * 6, 64 * 7], False)],
                         ids=["8", "8_and_a_token", "9", "ragged", "9_less_a_token", "6", "6_and_a_token", "6_and_7"])
def test_shortest_sequences_that_are_cut(V, lens, uniform, dtype):
    c = Case(lens, Hk=2, dk=64, dv=64, dtype=dtype, uniform=uniform, rough=True)
    c.check_forward(*c.forward(V))
    c.check_backward(c.backward(V))


@pytest.mark.parametrize("n", [1024, 1100, 2050])
def test_more_sequences_than_the_planning_threads(V, n):
    lens = [int(x) for x in np.random.default_rng(n).integers(0, 4, n)]
    lens[n - 20] = 64 * 17
    c = Case(lens, Hk=1, dk=32, dv=32, layout="tokens")
    c.check_forward(*c.forward(V))
    c.check_backward(c.backward(V))


def _guarded(t, value=7.0):
    """A tensor like t within a buffer of `value`, and the buffer's parts outside it."""
    import torch
    pad = 4096
    buf = torch.full((t.numel() + 2 * pad,), value, dtype=t.dtype, device="cuda")
    return buf[pad:pad + t.numel()].view(t.shape), (buf[:pad], buf[pad + t.numel():])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [dict(lens=[64 * 18], Hk=1, group=2, dk=128, dv=128),
                                  dict(lens=[64 * 18 + 1, 0, 100], Hk=1, group=3, dk=32, dv=64, layout="tokens"),
                                  dict(lens=[300, 70], Hk=4, dk=64, dv=128)], ids=["cut_128", "cut_32x64", "whole"])
def test_nothing_else_is_written(V, case, dtype):
    """Outputs and workspace within guarded buffers, inputs as they were."""
    import torch
    c = Case(dtype=dtype, **case)
    d = c.dev
    args = [d[x] for x in ("q", "k", "v", "g", "beta")]
    inputs = args + [d["do"], c.cu_dev] + c.states
    before = [t.clone() for t in inputs]
    works = [_guarded(torch.empty(V.delta_workspace(*args, cu_seqlens=c.cu_dev, layout=c.layout, backward=b),
                                  dtype=torch.uint8), 0x5a) for b in (False, True)]
    out, S = _guarded(d["v"]), _guarded(c.states[0])
    grads = [_guarded(t) for t in args + [c.states[0]]]
    c.check_forward(*c.forward(V, out=out[0], state_out=S[0], work=works[0][0]))
    c.check_backward(c.backward(V, outs=[t for t, _ in grads], work=works[1][0]))
    assert all((p == 7).all() for _, parts in grads + [out, S] for p in parts)
    assert all((p == 0x5a).all() for _, parts in works for p in parts)
    assert all(torch.equal(x, y) for x, y in zip(inputs, before))


@pytest.mark.parametrize("offsets", [[0, 200, 100, 300], [300, 0, 300, 0, 300], [0, 300, 0, 300, 0, 300, 0, 300]])
def test_decreasing_offsets_stay_inside(V, offsets):
    """A malformed list: nothing outside the tensors and the workspace is written, and what only a first sequence
    covers is right."""
    import torch
    c = Case(lens=[200, 100], Hk=2, dk=64, dv=64, state=False)
    want = c.forward(V)
    cu = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    d = c.dev
    args = [d[x] for x in ("q", "k", "v", "g", "beta")]
    out, guard = _guarded(d["v"])
    need = [V.delta_workspace(*args, cu_seqlens=cu, backward=b) for b in (False, True)]
    works = [_guarded(torch.empty(n, dtype=torch.uint8), 0x5a) for n in need]
    V.delta_forward(*args, cu_seqlens=cu, scale=c.scale, out=out, work=works[0][0])
    grads = [_guarded(t) for t in args]
    dS, dS_guard = _guarded(torch.empty(len(offsets) - 1, 2, 64, 64))
    V.delta_backward(d["do"], *args, cu_seqlens=cu, scale=c.scale, outs=[t for t, _ in grads] + [dS],
                     work=works[1][0])
    for parts in [guard, dS_guard] + [p for _, p in grads]:
        assert all((p == 7).all() for p in parts)
    assert all((p == 0x5a).all() for _, parts in works for p in parts)
    if offsets[1] == 200:
        assert torch.equal(out[:, :100], want[0][:, :100])


def test_tensors_past_32_bits(V):
    """The last sequence of tensors of more than 2^31 elements (heads layout), and of more than 2^31 bytes with a
    workspace of tens of GiB in the backward pass (tokens layout)."""
    import torch
    T = (1 << 20) + 200
    small = Case(lens=[200], Hk=1, dk=128, dv=128, seed=5)
    for H, layout in ((16, "heads"), (8, "tokens")):
        print(f"{H} heads of {T} tokens, {layout}", flush=True)
        torch.cuda.empty_cache()
        g = torch.Generator(device="cuda").manual_seed(2)
        shape = (H, T) if layout == "heads" else (T, H)

        def fill(d, last, scale):
            x = torch.empty(*shape, *d, dtype=last.dtype, device="cuda").normal_(0, scale, generator=g)
            part = x[:, -200:] if layout == "heads" else x[-200:].transpose(0, 1)
            part.copy_(last.cuda().expand_as(part))
            return x

        h = small.host
        q, k, v = fill((128,), h["q"], 128 ** -0.5), fill((128,), h["k"], 128 ** -0.5), fill((128,), h["v"], 1.0)
        gate, beta = fill((), h["g"], 0.0).add_(0), fill((), h["beta"], 0.0)
        cu = torch.tensor([0, T - 200, T], dtype=torch.int32, device="cuda")
        kw = dict(cu_seqlens=cu, layout=layout, scale=small.scale)
        tail = lambda x: (x[-1:, -200:] if layout == "heads" else x[-200:, -1:].transpose(0, 1))  # noqa: E731
        S = torch.stack([torch.zeros(H, 128, 128), small.S[0].expand(H, 128, 128)]).cuda()
        if layout == "heads":
            out, last = V.delta_forward(q, k, v, gate, beta, state=S, return_state=True, **kw)
            small.check_forward(tail(out).contiguous(), last[1:, -1:])
        else:
            dS = torch.stack([torch.zeros(H, 128, 128), small.dS[0].expand(H, 128, 128)]).cuda()
            do = fill((128,), h["do"], 1.0)
            grads = V.delta_backward(do, q, k, v, gate, beta, state=S, dstate=dS, **kw)
            small.check_backward([tail(x).contiguous() for x in grads[:5]] + [grads[5][1:, -1:]])
            del do, grads
        del q, k, v, gate, beta, S
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------------------------------------------------
# The recurrent form
# ---------------------------------------------------------------------------------------------------------------------

def _step_case(n, t, Hk, group, dk, dv, dtype, seed=0):
    import torch
    rng = np.random.default_rng(seed + n + 10 * t + dk)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Hv = Hk * group

    def unit(*s):
        x = rng.standard_normal(s)
        return torch.from_numpy(x / np.linalg.norm(x, axis=-1, keepdims=True)).to(dt)

    q, k = unit(n, t, Hk, dk), unit(n, t, Hk, dk)
    v = torch.from_numpy(rng.standard_normal((n, t, Hv, dv))).to(dt)
    g = torch.from_numpy(-rng.random((n, t, Hv)) ** 3 * 3).float()
    beta = torch.from_numpy(rng.random((n, t, Hv))).float()
    return q, k, v, g, beta


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,t,Hk,group,dk,dv", [(1, 1, 1, 1, 32, 32), (3, 1, 2, 2, 128, 128), (5, 3, 1, 3, 64, 128),
                                                (2, 7, 3, 1, 128, 32), (9, 2, 2, 1, 32, 128), (2, 1, 1, 1, 64, 64)])
def test_step(V, n, t, Hk, group, dk, dv, dtype):
    """Slots in any order, unused ones and rows of padding left alone."""
    import torch
    print(f"delta step n={n} t={t} Hk={Hk} group={group} {dk}x{dv} {dtype}", flush=True)
    q, k, v, g, beta = _step_case(n, t, Hk, group, dk, dv, dtype)
    g[0, 0, 0] = -np.inf
    slots = np.random.default_rng(n).permutation(n + 3)[:n]
    if n > 2:
        slots[1] = -1
    if n > 4:
        slots[3] = n + 3  # past the pool
    rng = np.random.default_rng(7)
    pool = torch.from_numpy(rng.standard_normal((n + 3, Hk * group, dv, dk))).float()
    state = pool.cuda()
    out = torch.full(v.shape, 5.0, dtype=v.dtype, device="cuda")
    scale = 0.25
    got = V.delta_step(q.cuda(), k.cuda(), v.cuda(), g.cuda(), beta.cuda(), state,
                       slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), scale=scale, out=out)
    assert got is out
    ref_state, ref = pool.double().numpy(), np.full(v.shape, 5.0)
    for i, s in enumerate(slots):
        if not 0 <= s < n + 3:
            continue
        for h in range(Hk * group):
            ref[i, :, h], ref_state[s, h] = D.delta_head(
                *(x[i, :, h // group].double().numpy() for x in (q, k)), v[i, :, h].double().numpy(),
                g[i, :, h].double().numpy(), beta[i, :, h].double().numpy(), ref_state[s, h], scale)
    assert _err(from_device(out), ref) <= (2.0 ** -8 if dtype == "bf16" else TOL_OUT["f32"])
    assert _err(from_device(state), ref_state) <= TOL_OUT["f32"]
    idle = [s for s in range(n + 3) if s not in slots]
    assert torch.equal(state[idle].cpu(), pool[idle])
    for i, s in enumerate(slots):
        if not 0 <= s < n + 3:
            assert (out[i] == 5).all()


def test_step_without_slots_and_errors(V):
    import torch
    q, k, v, g, beta = (x.cuda() for x in _step_case(2, 1, 1, 1, 32, 32, "f32"))
    state = torch.zeros(3, 1, 32, 32, device="cuda")
    V.delta_step(q, k, v, g, beta, state)
    # From zero: S = beta v k^T.
    want = (beta[:, 0, :, None] * v[:, 0])[..., None] * k[:, 0, :, None, :]
    assert _err(from_device(state[:2]), from_device(want)) <= 4 * 2.0 ** -24
    assert (state[2] == 0).all()
    for kw in (dict(state=state[:1]), dict(slots=torch.zeros(2, device="cuda")), dict(state=state.double()),
               dict(out=torch.empty(2, 1, 1, 31, device="cuda"))):
        with pytest.raises(ValueError):
            V.delta_step(q, k, v, g, beta, **{"state": state, **kw})


def test_step_far_into_the_pool(V):
    """A slot whose state begins past 2^32 bytes."""
    import torch
    q, k, v, g, beta = (x.cuda() for x in _step_case(2, 1, 8, 2, 128, 128, "bf16"))
    per = 16 * 128 * 128
    n = (1 << 30) // per + 9
    pool = torch.zeros(n, 16, 128, 128, device="cuda")
    near = torch.randn(2, 16, 128, 128, device="cuda")
    pool[-1], pool[3] = near[0], near[1]
    out = V.delta_step(q, k, v, g, beta, pool, slots=torch.tensor([n - 1, 3], dtype=torch.int32, device="cuda"))
    want = V.delta_step(q, k, v, g, beta, near)
    assert torch.equal(out, want) and torch.equal(pool[-1], near[0]) and torch.equal(pool[3], near[1])


def test_step_in_a_graph(V):
    import torch
    q, k, v, g, beta = (x.cuda() for x in _step_case(4, 2, 2, 2, 64, 64, "bf16"))
    first = torch.randn(4, 4, 64, 64, device="cuda")
    state = first.clone()
    graph = torch.cuda.CUDAGraph()
    V.delta_step(q, k, v, g, beta, state.clone())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = V.delta_step(q, k, v, g, beta, state)
    eager = first.clone()
    for turn in range(3):
        graph.replay()
        want = V.delta_step(q, k, v, g, beta, eager)
        torch.cuda.synchronize()
        assert torch.equal(state, eager) and torch.equal(out, want), turn


# ---------------------------------------------------------------------------------------------------------------------
# Together, as a streaming video model uses them
# ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_then_steps(V, dtype):
    """A prompt through the chunk-wise form and the stream's further tokens through the recurrent one, on the state
    that the first left, are the whole stream in one call."""
    import torch
    c = Case(lens=[150, 150], uniform=True, Hk=2, group=2, dk=64, dv=64, dtype=dtype, layout="tokens", state=False)
    d, cut = c.dev, 143
    part = [d[x][:, :cut].contiguous() for x in ("q", "k", "v", "g", "beta")]
    out, S = V.delta_forward(*part, layout="tokens", scale=c.scale, return_state=True)
    outs = [out]
    for t0, t1 in ((143, 144), (144, 147), (147, 150)):
        step = [d[x][:, t0:t1].contiguous() for x in ("q", "k", "v", "g", "beta")]
        outs.append(V.delta_step(*step, S, scale=c.scale))
    c.check_forward(torch.cat(outs, 1), S)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotated_projections_through_the_rule_and_back(V, dtype):
    """q and k slices of a fused projection, rotated by their grid positions and L2-mapped, through the rule, and the
    loss's gradient back to the projection: against the oracle's chain in 64 bits on the same stored values."""
    import torch
    B, gh, gw, F, H, d = 2, 3, 5, 5, 2, 64
    L, axes, scale = gh * gw * F, (8, 12, 12), 0.5
    rng = np.random.default_rng(3)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    qkv = torch.from_numpy(rng.standard_normal((B, L, 3 * H * d))).to(dt)
    f = torch.from_numpy(np.concatenate([100.0 ** (-np.arange(a) / a) for a in axes])).float()
    g = torch.from_numpy(-rng.random((B, H, L)) * 0.3).float()
    beta = torch.from_numpy(rng.random((B, H, L))).float()
    do = torch.from_numpy(rng.standard_normal((B, H, L, d))).to(dt)

    x = qkv.cuda()
    opts = dict(grid=(gh, gw), frame_offset=2, l2=True)
    qk = V.rope(x[:, :, :2 * H * d], f.cuda(), axes, 2 * H, **opts).view(B, 2, H, L, d)
    q, k = qk[:, 0].contiguous(), qk[:, 1].contiguous()
    v = x[:, :, 2 * H * d:].unflatten(2, (H, d)).transpose(1, 2).contiguous()
    out = V.delta_forward(q, k, v, g.cuda(), beta.cuda(), scale=scale)
    dq, dk, dv, dg, dbeta, _ = V.delta_backward(do.cuda(), q, k, v, g.cuda(), beta.cuda(), scale=scale)
    dx = torch.empty_like(x)
    dqk = torch.stack([dq, dk], 1).view(B * 2 * H, L, d)
    V.rope_backward(dqk, f.cuda(), axes, 2 * H, x=x[:, :, :2 * H * d], out=dx[:, :, :2 * H * d], **opts)
    dx[:, :, 2 * H * d:] = dv.transpose(1, 2).flatten(2)

    pos = D.grid_positions(L, gh, gw, 2)
    ref_out, ref_dx = np.zeros((B, H, L, d)), np.zeros((B, L, 3 * H * d))
    ref_dg, ref_db = np.zeros((B, H, L)), np.zeros((B, H, L))
    for b in range(B):
        for h in range(H):
            xs = [qkv[b, :, (i * H + h) * d:(i * H + h + 1) * d].double().numpy() for i in range(3)]
            rq, rk = (D.rope_head(z, pos, f.numpy(), axes, True, True) for z in xs[:2])
            gb, bb = g[b, h].double().numpy(), beta[b, h].double().numpy()
            zero = np.zeros((d, d))
            ref_out[b, h], _ = D.delta_head(rq, rk, xs[2], gb, bb, zero, scale)
            r = D.delta_head_backward(do[b, h].double().numpy(), zero, rq, rk, xs[2], gb, bb, zero, scale)
            for i in range(2):
                r_in = D.rope_head_backward(r[i], xs[i], pos, f.numpy(), axes, True, True)
                ref_dx[b, :, (i * H + h) * d:(i * H + h + 1) * d] = r_in
            ref_dx[b, :, (2 * H + h) * d:(2 * H + h + 1) * d] = r[2]
            ref_dg[b, h], ref_db[b, h] = r[3], r[4]
    # The rotated q and k are stored once more (bf16: 2^-8 each), and the gradients between the two calls; the
    # gates' gradients then see rounded q and k as well.
    tol = {"bf16": 8 * 2.0 ** -8, "f32": 2 * TOL_OUT["f32"]}[dtype]
    for got, want in ((out, ref_out), (dx, ref_dx), (dg, ref_dg), (dbeta, ref_db)):
        assert _err(from_device(got), want) <= tol
