"""GPU parity of the cross attention to an encoder's states (cross_forward,
cross_backward, cross_step) against the fp64 oracle.

Each element of each output is held to the bound that its own roundings leave
(oracle/cross_oracle.py, cross_bounds): the storage type's where weights, score
gradients and outputs are rounded once, fp32's in sums and exponentials.
"""
import numpy as np
import pytest

import oracle.cross_oracle as X
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
    same = np.isneginf(want) & np.isneginf(got)
    err = np.where(same, 0.0, np.abs(got - np.where(same, 0.0, want)))
    err = np.where(same, 0.0, err)
    # 1e-30: subnormal outputs are flushed.
    ok = err <= bound + 1e-30
    assert ok.all(), (what, int((~ok).sum()), float(np.nanmax(err / (bound + 1e-30))), np.argwhere(~ok)[:4].tolist())


class Case:
    """Sequences on the host (the stored values, in 64 bits) and their tensors on the device."""

    def __init__(self, lq, lk, Hq=2, Hk=2, d=64, dtype="bf16", layout="tokens", kv_layout=None, out_layout=None, lens=None,
                 mask=None, packed=None, scale=None, fused=False, lead=0, tail=0, spread=1.0, seed=0):
        import torch
        rng = np.random.default_rng(seed + 31 * sum(lq) + sum(lk) + d)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.half, self.dtype = HALF[dtype], dtype
        self.lq, self.lk, self.n, self.d, self.Hq, self.Hk = lq, lk, len(lq), d, Hq, Hk
        self.layout, self.kv_layout, self.out_layout = layout, kv_layout or layout, out_layout or layout
        self.packed = len(set(lq)) > 1 or len(set(lk)) > 1 if packed is None else packed
        self.scale = d ** -0.5 if scale is None else scale
        self.lead, self.tail = lead, tail
        self.T, self.S = sum(lq) + lead + tail, sum(lk) + lead + tail

        def values(total, H, by):
            x = torch.from_numpy(by * rng.standard_normal((total, H, d))).to(self.dt)
            return x, x.double().numpy()

        (q, self.q), (k, self.k), (v, self.v) = values(self.T, Hq, spread), values(self.S, Hk, 1.0), values(self.S, Hk, 1.0)
        do, self.do = values(self.T, Hq, 1.0)
        self.cq = lead + np.concatenate([[0], np.cumsum(lq)])
        self.ck = lead + np.concatenate([[0], np.cumsum(lk)])
        seen = np.ones(self.S, bool)
        if mask == "holes":
            seen = rng.random(self.S) < 0.7
        elif mask == "none":
            seen[:] = False
        elif mask == "first":  # nothing of the first sequence
            seen[self.ck[0]:self.ck[1]] = False
        elif mask == "left":  # padding in front
            for i in range(self.n):
                seen[self.ck[i]:self.ck[i] + 2 * lk[i] // 3] = False
        self.mask = torch.from_numpy(seen.copy()) if mask else None
        self.k_lens = None
        if lens is not None:
            self.k_lens = torch.tensor(lens, dtype=torch.int32)
            for i, m in enumerate(lens):
                seen[self.ck[i] + min(max(m, 0), lk[i]):self.ck[i + 1]] = False
        self.seen = seen
        hidden = torch.from_numpy(~seen)
        inside = torch.zeros(self.S, dtype=torch.bool)
        inside[self.ck[0]:self.ck[-1]] = True
        hidden &= inside
        # What stands in places that are not seen changes nothing.
        k[hidden], v[hidden] = float("inf"), float("nan")
        self.dev = dict(q=self._place(q, self.layout, Hq, fused and 3), k=self._place(k, self.kv_layout, Hk, fused and 2),
                        v=self._place(v, self.kv_layout, Hk, fused and 2), dout=self._place(do, self.out_layout, Hq, 0))

    def _place(self, x, layout, H, fused):
        """The [tokens, H, d] values as the call takes them."""
        import torch
        if not self.packed:
            x = x.unflatten(0, (self.n, -1))
        if layout == "heads":
            return x.transpose(-3, -2).contiguous().cuda()
        if fused:
            wide = torch.full(x.shape[:-2] + (fused, H, self.d), 7.0, dtype=self.dt)
            wide[..., 1, :, :] = x
            return wide.cuda()[..., 1, :, :]
        return x.cuda()

    def options(self):
        import torch
        o = dict(layout=self.layout, kv_layout=self.kv_layout, out_layout=self.out_layout, scale=self.scale)
        if self.packed:
            o["cu_q"] = torch.tensor(self.cq, dtype=torch.int32, device="cuda")
            o["cu_k"] = torch.tensor(self.ck, dtype=torch.int32, device="cuda")
        if self.mask is not None:
            o["k_mask"] = (self.mask if self.packed else self.mask.unflatten(0, (self.n, -1))).cuda()
        if self.k_lens is not None:
            o["k_lens"] = self.k_lens.cuda()
        return o

    def tokens(self, t, layout):
        """[tokens, H, d] in 64 bits of a result."""
        x = from_device(t.contiguous())
        if layout == "heads":
            x = np.swapaxes(x, -3, -2)
        return x.reshape(-1, *x.shape[-2:])

    def lse_tokens(self, t):
        x = np.swapaxes(from_device(t), -1, -2)
        return x.reshape(-1, self.Hq)

    def check(self, out, lse, grads=None):
        out, lse = self.tokens(out, self.out_layout), self.lse_tokens(lse)
        if grads is not None:
            dq, dk, dv = self.tokens(grads[0], self.layout), self.tokens(grads[1], self.kv_layout), self.tokens(grads[2], self.kv_layout)
        for i in range(self.n):
            r, c = slice(self.cq[i], self.cq[i + 1]), slice(self.ck[i], self.ck[i + 1])
            a = (self.q[r], self.k[c], self.v[c], self.seen[c], self.scale)
            if grads is None:
                want, bound = X.cross_sequence(*a), X.cross_bounds(*a, self.half)
                got = (out[r], lse[r])
            else:
                want, bound = X.cross_sequence(*a, self.do[r]), X.cross_bounds(*a, self.half, self.do[r])
                got = (out[r], lse[r], dq[r], dk[c], dv[c])
            for g, w, b, name in zip(got, want, bound, ("out", "lse", "dq", "dk", "dv")):
                _hold(g, w, b, (name, i))


CASES = {
    "one": dict(lq=[1], lk=[1]),
    "one_of_many": dict(lq=[1], lk=[1000], Hq=4, Hk=1, d=128),
    "many_of_one": dict(lq=[300], lk=[1], d=32),
    "rows_32": dict(lq=[32], lk=[65], d=128),
    "rows_33": dict(lq=[33], lk=[63], d=128),
    "rows_129": dict(lq=[129, 129], lk=[64, 64], layout="heads"),
    "rows_127_group": dict(lq=[43], lk=[129], Hq=6, Hk=2, layout="heads", kv_layout="tokens"),
    "group_odd": dict(lq=[50, 50], lk=[77, 77], Hq=15, Hk=3, d=32, layout="tokens", kv_layout="heads", out_layout="heads"),
    "packed": dict(lq=[70, 0, 1, 200, 33], lk=[130, 5, 64, 1, 90], Hq=4, Hk=2, d=128, lead=3, tail=5),
    "packed_heads": dict(lq=[5, 260, 0, 40], lk=[300, 0, 7, 129], Hq=4, Hk=4, layout="heads", lead=1, tail=2),
    "packed_many": dict(lq=[(7 * i) % 23 for i in range(70)], lk=[(5 * i) % 31 for i in range(70)], d=32),
    # Many rows each: up to 63 sequences are taken longest first, more in their own order.
    "packed_63": dict(lq=[(37 * i) % 101 for i in range(63)], lk=[(29 * i) % 83 for i in range(63)], Hq=3, Hk=1, d=32, lead=2, tail=2),
    "packed_64": dict(lq=[(37 * i) % 101 for i in range(64)], lk=[(29 * i) % 83 for i in range(64)], Hq=3, Hk=1, d=32, lead=2, tail=2),
    "packed_alike": dict(lq=[130] * 5, lk=[65] * 5, Hq=2, Hk=1, d=64, packed=True, mask="holes"),
    "packed_rows_of_one": dict(lq=[400, 1, 0, 900], lk=[1, 700, 300, 64], Hq=5, Hk=5, d=128, lens=[1, 650, 300, 64]),
    "few_short": dict(lq=[2, 2], lk=[250, 250], Hq=4, Hk=2, d=128, mask="holes", lens=[250, 100]),
    "few_of_many": dict(lq=[3] * 140, lk=[70] * 140, Hq=2, Hk=2, d=32, mask="left"),
    "few_long": dict(lq=[9, 9], lk=[2500, 2500], Hq=2, Hk=1, d=64),
    "some_long": dict(lq=[100], lk=[3001], Hq=1, Hk=1, d=128, layout="heads"),
    "lens": dict(lq=[40, 40, 40, 40], lk=[100, 100, 100, 100], lens=[0, 1, 64, 1000], d=128),
    "lens_below": dict(lq=[200, 200], lk=[70, 70], lens=[-5, 70], layout="heads"),
    "holes": dict(lq=[150, 150], lk=[200, 200], mask="holes", Hq=4, Hk=2, d=128),
    "holes_few": dict(lq=[3, 3], lk=[700, 700], mask="holes", Hq=4, Hk=2, d=128),
    "left": dict(lq=[64, 64], lk=[150, 150], mask="left"),
    "left_few": dict(lq=[2, 30], lk=[450, 3], mask="left", d=32),
    "nothing": dict(lq=[140], lk=[90], mask="none"),
    "first_nothing": dict(lq=[4, 140, 1], lk=[90, 20, 300], mask="first", lens=[5, 20, 299], lead=2, tail=1),
    "fused": dict(lq=[60, 60], lk=[81, 81], Hq=4, Hk=2, d=64, fused=True),
    "fused_packed": dict(lq=[60, 7], lk=[81, 140], Hq=2, Hk=2, d=128, fused=True, mask="holes", lead=1, tail=1),
    "scale_below_0": dict(lq=[90], lk=[100], scale=-0.3, d=128),
    "scale_0": dict(lq=[90, 2], lk=[100, 65], scale=0.0, mask="holes"),
    "peaked": dict(lq=[130], lk=[300], scale=1.0, spread=3.0, d=64),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_forward_and_gradients(V, name, dtype):
    c = Case(dtype=dtype, **CASES[name])
    print(name, dtype, flush=True)
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    grads = V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)
    c.check(out, lse, grads)


ALONE = {
    "one_state": dict(lq=[70, 5], lk=[1, 1], Hq=4, Hk=2, d=128),
    "lens": dict(lq=[40, 40], lk=[120, 120], lens=[1, 1], d=64, layout="heads"),
    "masked": dict(lq=[200, 3, 40], lk=[128, 70, 65], Hq=3, Hk=1, d=32),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ALONE)
def test_a_state_seen_alone_has_no_gradient_of_scores(V, name, dtype):
    """A softmax over one state is constant: dq and dk are zeros, not what roundings leave."""
    import torch
    c = Case(dtype=dtype, **ALONE[name])
    if name == "masked":  # one state of each sequence: the first, the last of the first tile, the last
        at = [0, c.ck[1] + 63, c.ck[3] - 1]
        c.seen[:] = False
        c.seen[at] = True
        c.mask = torch.from_numpy(c.seen.copy())
        hidden = torch.from_numpy(~c.seen).cuda()
        c.dev["k"][hidden], c.dev["v"][hidden] = float("nan"), float("inf")
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    dq, dk, dv = V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)
    c.check(out, lse, (dq, dk, dv))
    assert not dq.any() and not dk.any()


@pytest.mark.parametrize("lk", [2, 5, 30, 128, 129, 600])
def test_gradients_of_few_states_keep_their_norm(V, lk):
    """What roundings leave of a gradient's norm.  One to bf16 is off by 2^-8 of a value's power of two at most, evenly, so by
    2^-8 / sqrt(3) of that in the root mean square, and that is 0.73 of the values' own: 0.0017 of a vector's norm.  dq and
    dk have two (score gradients, result), dv two (weights, result): 0.0017 sqrt(2) = 0.0024.  D taken from a rounded
    output is a third, as large where few states share the weight (0.0029): a third of its square at most may stay."""
    import torch
    c = Case(lq=[130] * 4, lk=[lk] * 4, Hq=4, Hk=4, d=128, spread=1.5)
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    grads = V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)
    dq, dk, dv = (c.tokens(x, "tokens") for x in grads)
    off = np.zeros((3, 2))
    for i in range(c.n):
        r, s = slice(c.cq[i], c.cq[i + 1]), slice(c.ck[i], c.ck[i + 1])
        want = X.cross_sequence(c.q[r], c.k[s], c.v[s], c.seen[s], c.scale, c.do[r])[2:]
        for x, g, w in zip(off, (dq[r], dk[s], dv[s]), want):
            x += (np.sum((g - w) ** 2), np.sum(w ** 2))
    assert (np.sqrt(off[:, 0] / off[:, 1]) < 0.0026).all(), np.sqrt(off[:, 0] / off[:, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lq, lk, lens", [([70, 3, 0, 200], [90] * 4, [90, 1, 40, 65]), ([2, 9, 0, 5], [300] * 4, [0, 300, 7, 150]),
                                          ([130] * 3, [200, 0, 61], None), ([4] * 3, [700, 1, 33], None)])
def test_packed_on_one_side(V, lq, lk, lens, dtype):
    """Packed queries and padded states, and the other way round."""
    c = Case(lq=lq, lk=lk, Hq=4, Hk=2, d=64, lens=lens, mask="holes", packed=True, dtype=dtype)
    d, o = c.dev, c.options()
    if len(set(lk)) == 1:
        del o["cu_k"]
        d["k"], d["v"], o["k_mask"] = (x.unflatten(0, (len(lk), -1)) for x in (d["k"], d["v"], o["k_mask"]))
    else:
        del o["cu_q"]
        d["q"], d["dout"] = (x.unflatten(0, (len(lq), -1)) for x in (d["q"], d["dout"]))
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    c.check(out, lse, V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o))


def test_rows_outside_sequences_are_left(V):
    import torch
    c = Case(lq=[5, 40], lk=[70, 3], lead=4, tail=6, Hq=2, Hk=1)
    d, o = c.dev, c.options()
    out = torch.full_like(d["q"], 3.0)
    lse = torch.full((c.Hq, c.T), 3.0, device="cuda")
    V.cross_forward(d["q"], d["k"], d["v"], out=out, lse=lse, **o)
    grads = [torch.full_like(d[x], 3.0) for x in ("q", "k", "v")]
    V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, outs=grads, **o)
    c.check(out, lse, grads)
    for t, cu in ((out, c.cq), (grads[0], c.cq), (grads[1], c.ck), (grads[2], c.ck)):
        assert (t[:cu[0]] == 3.0).all() and (t[cu[-1]:] == 3.0).all()
    assert (lse[:, :c.cq[0]] == 3.0).all() and (lse[:, c.cq[-1]:] == 3.0).all()


def test_few_rows_outside_sequences_are_left(V):
    """... where ranges of the states are joined."""
    import torch
    c = Case(lq=[5, 4], lk=[1700, 900], lead=4, tail=6, Hq=2, Hk=1)
    d, o = c.dev, c.options()
    assert V.cross_workspace(d["q"], d["k"], d["v"], o["cu_q"], o["cu_k"], layout="tokens") > 0
    out = torch.full_like(d["q"], 3.0)
    lse = torch.full((c.Hq, c.T), 3.0, device="cuda")
    V.cross_forward(d["q"], d["k"], d["v"], out=out, lse=lse, **o)
    grads = [torch.full_like(d[x], 3.0) for x in ("q", "k", "v")]
    V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, outs=grads, **o)
    c.check(out, lse, grads)
    for t, cu in ((out, c.cq), (grads[0], c.cq), (grads[1], c.ck), (grads[2], c.ck)):
        assert (t[:cu[0]] == 3.0).all() and (t[cu[-1]:] == 3.0).all()
    assert (lse[:, :c.cq[0]] == 3.0).all() and (lse[:, c.cq[-1]:] == 3.0).all()


def test_fused_gradients_leave_what_lies_between(V):
    import torch
    c = Case(lq=[30, 30], lk=[50, 50], Hq=2, Hk=2, d=64)
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    kv = torch.full((2, 50, 3, 2, 64), 5.0, dtype=c.dt, device="cuda")
    dq = torch.full((2, 30, 2, 2, 64), 5.0, dtype=c.dt, device="cuda")
    outs = (dq[:, :, 1], kv[:, :, 0], kv[:, :, 2])
    V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, outs=outs, **o)
    c.check(out, lse, outs)
    assert (kv[:, :, 1] == 5.0).all() and (dq[:, :, 0] == 5.0).all()


def _step_case(V, n, t, m, S, Hq, Hk, d, dtype, kv_layout, lens=None, mask=None, slots=None, fused=False, seed=0):
    import torch
    rng = np.random.default_rng(seed + n + S + d)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.from_numpy(rng.standard_normal((n, t, Hq, d))).to(dt)
    k, v = (torch.from_numpy(rng.standard_normal((m, S, Hk, d))).to(dt) for _ in range(2))
    seen = np.ones((m, S), bool)
    if mask:
        seen = rng.random((m, S)) < 0.6
        seen[m // 2] = False
    kw = dict(k_mask=torch.from_numpy(seen.copy()).cuda()) if mask else {}
    if lens is not None:
        kw["k_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        for i, x in enumerate(lens):
            seen[i, max(x, 0):] = False
    kd, vd = k.double().numpy(), v.double().numpy()
    hidden = torch.from_numpy(~seen)
    k[hidden], v[hidden] = float("nan"), float("inf")
    if fused:
        kv = torch.stack([k, v], 2).cuda()
        kc, vc = kv[:, :, 0], kv[:, :, 1]
    elif kv_layout == "heads":
        kc, vc = (x.transpose(1, 2).contiguous().cuda() for x in (k, v))
    else:
        kc, vc = k.cuda(), v.cuda()
    where = list(range(n)) if slots is None else slots
    out = torch.full((n, t, Hq, d), 9.0, dtype=dt, device="cuda")
    V.cross_step(q.cuda(), kc, vc, slots=None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda"),
                 kv_layout=kv_layout, out=out, **kw)
    got = from_device(out)
    for i, s in enumerate(where):
        if s < 0 or s >= m:
            assert (got[i] == 9.0).all()
            continue
        a = (q[i].double().numpy(), kd[s], vd[s], seen[s], d ** -0.5)
        _hold(got[i], X.cross_sequence(*a)[0], X.cross_bounds(*a, HALF[dtype])[0], (i, s))


STEPS = {
    "one": dict(n=1, t=1, m=1, S=1, Hq=1, Hk=1, d=32, kv_layout="tokens"),
    "prompt": dict(n=1, t=1, m=4, S=512, Hq=16, Hk=16, d=128, kv_layout="tokens", slots=[2]),
    "shared": dict(n=9, t=1, m=5, S=700, Hq=8, Hk=2, d=128, kv_layout="tokens", slots=[4, 0, 0, -1, 2, 5, 4, 1 << 30, 3],
                   lens=[700, 1, 0, 333, 64]),
    "tokens": dict(n=3, t=5, m=3, S=130, Hq=8, Hk=2, d=64, kv_layout="heads", lens=[130, 129, 1]),
    "many_rows": dict(n=2, t=40, m=2, S=70, Hq=4, Hk=2, d=64, kv_layout="heads"),
    "mask": dict(n=4, t=2, m=4, S=260, Hq=4, Hk=4, d=128, kv_layout="tokens", mask=True),
    "mask_lens": dict(n=4, t=1, m=6, S=1030, Hq=4, Hk=1, d=64, kv_layout="heads", mask=True, lens=[5, 1030, 600, 2000, 0, 31],
                      slots=[0, 1, 3, 2]),
    "fused": dict(n=3, t=1, m=3, S=90, Hq=6, Hk=3, d=32, kv_layout="tokens", fused=True),
    "short": dict(n=2, t=3, m=2, S=256, Hq=8, Hk=2, d=128, kv_layout="heads", mask=True, lens=[256, 97]),
    "short_64": dict(n=2, t=1, m=2, S=512, Hq=8, Hk=2, d=64, kv_layout="tokens", mask=True, lens=[1, 512]),
    "unsplit": dict(n=40, t=1, m=40, S=300, Hq=16, Hk=8, d=64, kv_layout="tokens", mask=True),
    "many": dict(n=300, t=1, m=300, S=33, Hq=2, Hk=1, d=32, kv_layout="tokens"),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", STEPS)
def test_step(V, name, dtype):
    print(name, dtype, flush=True)
    _step_case(V, dtype=dtype, **STEPS[name])


def test_step_is_the_whole_sequence(V):
    """Tokens one at a time give what the whole sequence gives, up to both calls' roundings."""
    import torch
    c = Case(lq=[6, 6], lk=[200, 200], Hq=4, Hk=2, d=64)
    d = c.dev
    whole = V.cross_forward(d["q"], d["k"], d["v"], layout="tokens")
    steps = torch.cat([V.cross_step(d["q"][:, t:t + 1].contiguous(), d["k"], d["v"]) for t in range(6)], 1)
    for i in range(2):
        a = (c.q[c.cq[i]:c.cq[i + 1]], c.k[c.ck[i]:c.ck[i + 1]], c.v[c.ck[i]:c.ck[i + 1]], np.ones(200, bool), c.scale)
        bound = X.cross_bounds(*a, c.half)[0]
        _hold(from_device(steps[i]), from_device(whole[i]), 2 * bound, i)


def test_same_bits_again(V):
    import torch
    c = Case(lq=[70, 0, 1, 200], lk=[1300, 5, 64, 700], Hq=4, Hk=2, d=128, mask="holes")
    d, o = c.dev, c.options()
    first = None
    for _ in range(5):
        out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
        got = [out, lse, *V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)]
        got = [t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).clone() for t in got]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_garbage_in_work_and_outputs(V):
    """Nothing that a buffer held before comes through."""
    import torch
    c = Case(lq=[4, 4], lk=[1000, 1000], Hq=2, Hk=1, d=64, lens=[0, 900])
    d, o = c.dev, c.options()
    n = V.cross_workspace(d["q"], d["k"], d["v"], layout="tokens")
    m = V.cross_workspace(d["q"], d["k"], d["v"], layout="tokens", backward=True)
    assert n > 0 and m > 0
    work = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # NaN
    nan = [torch.full_like(d[x], float("nan")) for x in ("q", "k", "v")]
    out = torch.full_like(d["q"], float("nan"))
    _, lse = V.cross_forward(d["q"], d["k"], d["v"], out=out, return_lse=True, work=work, **o)
    V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, outs=nan,
                     work=torch.full((m,), 255, dtype=torch.uint8, device="cuda"), **o)
    c.check(out, lse, nan)


def test_captured_and_replayed(V):
    """A graph of a forward and a backward pass, replayed on other inputs, with eager work between."""
    import torch
    c = Case(lq=[5, 40], lk=[1200, 300], Hq=4, Hk=2, d=64, mask="holes")
    e = Case(lq=[5, 40], lk=[1200, 300], Hq=4, Hk=2, d=64, mask="holes", seed=9)
    o, buf = c.options(), {x: t.clone() for x, t in c.dev.items()}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def run():
        out, lse = V.cross_forward(buf["q"], buf["k"], buf["v"], return_lse=True, **o)
        return out, lse, V.cross_backward(buf["dout"], buf["q"], buf["k"], buf["v"], out, lse, **o)

    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out, lse, grads = run()
    for case in (c, e, c, e):
        for x, t in case.dev.items():
            buf[x].copy_(t)
        o["k_mask"].copy_(case.options()["k_mask"])
        g.replay()
        torch.cuda.synchronize()
        case.check(out, lse, grads)
        run()
        torch.cuda.synchronize()


def test_two_streams_at_once(V):
    import torch
    cases = [Case(lq=[3, 3], lk=[3000, 3000], Hq=2, Hk=1, d=64, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(4):
        for i, (c, s) in enumerate(zip(cases, streams)):
            got[i] = V.cross_forward(c.dev["q"], c.dev["k"], c.dev["v"], return_lse=True, stream=s, **c.options())
    torch.cuda.synchronize()
    for c, (out, lse) in zip(cases, got):
        c.check(out, lse)


def test_offsets_out_of_order(V):
    """Offsets that decrease or lie outside the tensors: values are undefined, what is around the tensors is not touched."""
    import torch
    guard, T, S, H, d = 512, 90, 300, 2, 32
    for cq, ck in (([0, 90, 30, 90], [0, 300, 10, 300]), ([-5, 40, 1000, 2000], [7, 3, -9, 1 << 30]),
                   ([90, 60, 30, 0], [300, 200, 100, 0]), ([0, 0, 0, 0], [0, 0, 0, 0])):
        q, k, v, do = (torch.randn(n, H, d, device="cuda").bfloat16() for n in (T, S, S, T))
        o = dict(layout="tokens", cu_q=torch.tensor(cq, dtype=torch.int32, device="cuda"),
                 cu_k=torch.tensor(ck, dtype=torch.int32, device="cuda"))
        outs = []
        for n in (T, T, S, S):
            wide = torch.full((n + 2 * guard, H, d), 5.0, device="cuda", dtype=torch.bfloat16)
            outs.append((wide, wide[guard:guard + n]))
        lse = torch.zeros(H, T, device="cuda")
        V.cross_forward(q, k, v, out=outs[0][1], lse=lse, **o)
        V.cross_backward(do, q, k, v, outs[0][1], lse, outs=[w[1] for w in outs[1:]], **o)
        torch.cuda.synchronize()
        for wide, _ in outs:
            assert (wide[:guard] == 5.0).all() and (wide[-guard:] == 5.0).all()


def test_states_past_32_bits_of_offsets(V):
    """A pool of 5 GB: its last slots are read."""
    import torch
    m, S, H, d = 40, 16400, 32, 128
    k = torch.zeros(m, S, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[-1, :200].normal_(), v[-1, :200].normal_()
    q = torch.randn(1, 1, H, d, device="cuda").bfloat16()
    lens = torch.full((m,), 200, dtype=torch.int32, device="cuda")
    out = V.cross_step(q, k, v, k_lens=lens, slots=torch.tensor([m - 1], dtype=torch.int32, device="cuda"))
    a = (from_device(q[0]), from_device(k[-1, :200]), from_device(v[-1, :200]), np.ones(200, bool), d ** -0.5)
    _hold(from_device(out[0]), X.cross_sequence(*a)[0], X.cross_bounds(*a, 2.0 ** -8)[0], "last slot")


def test_refusals_of_the_binding(V):
    import torch
    c = Case(lq=[4, 4], lk=[6, 6])
    d = c.dev
    q, k, v = d["q"], d["k"], d["v"]
    for kw in (dict(layout="rows"), dict(out_layout="rows"), dict(kv_layout="heads"), dict(k_lens=torch.zeros(2, device="cuda")),
               dict(k_lens=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(k_mask=torch.ones(2, 6, device="cuda")),
               dict(k_mask=torch.ones(12, dtype=torch.bool, device="cuda")),
               dict(cu_q=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(out=torch.zeros(2, 4, 2, 64, device="cuda")),
               dict(work=torch.zeros(4, device="cuda")), dict(lse=torch.zeros(2, 4, 2, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            V.cross_forward(q, k, v, **{"layout": "tokens", **kw})
    with pytest.raises(ValueError):
        V.cross_forward(q, k[:1], v[:1], layout="tokens")
    with pytest.raises(ValueError):
        V.cross_forward(q, k, v[:, :, :1], layout="tokens")
    with pytest.raises(ValueError):
        V.cross_forward(q.float(), k, v, layout="tokens")
    with pytest.raises(ValueError):
        V.cross_forward(q[..., :48].contiguous(), k[..., :48].contiguous(), v[..., :48].contiguous(), layout="tokens")
    with pytest.raises(ValueError):
        V.cross_forward(q[:, :0], k, v, layout="tokens")
    with pytest.raises(ValueError):
        V.cross_forward(q, k[:, :0], v[:, :0], layout="tokens")
    out, lse = V.cross_forward(q, k, v, layout="tokens", return_lse=True)
    with pytest.raises(ValueError):
        V.cross_backward(d["dout"], q, k, v, out, lse[:1], layout="tokens")
    with pytest.raises(ValueError):
        V.cross_backward(d["dout"], q, k, v, out, lse, layout="tokens", outs=(q.clone(), k.clone()))
    g = k.clone()
    with pytest.raises(ValueError):
        V.cross_backward(d["dout"], q, k, v, out, lse, layout="tokens", outs=(q.clone(), g, g))
    with pytest.raises(ValueError):
        V.cross_step(q, k, v, slots=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        V.cross_step(torch.cat([q, q]), k, v)  # four sequences, two slots


@pytest.mark.parametrize("S", [2, 30, 256])
def test_steps_over_few_states_keep_their_norm(V, S):
    """Weights in two parts leave the output's own rounding: 0.0017 of its norm (as above), and of a sum over thousands of
    values no more than a tenth beyond."""
    import torch
    rng = np.random.default_rng(S)
    q, k, v = (torch.from_numpy(rng.standard_normal((2, n, 4, 128))).bfloat16() for n in (2, S, S))
    got = from_device(V.cross_step(q.cuda(), k.cuda(), v.cuda()))
    off = total = 0.0
    for i in range(2):
        want = X.cross_sequence(*(x[i].double().numpy() for x in (q, k, v)), np.ones(S, bool), 128 ** -0.5)[0]
        off, total = off + np.sum((got[i] - want) ** 2), total + np.sum(want ** 2)
    assert np.sqrt(off / total) < 0.0019
