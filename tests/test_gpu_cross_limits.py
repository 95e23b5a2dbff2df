"""The cross attention at the ends of what its index arithmetic takes: many query heads
to a key head (groups that are no power of two, larger than a tile's rows, the largest),
and tensors whose heads or rows are more than 2^31 bytes from the first."""
import numpy as np
import pytest

import oracle.cross_oracle as X
from test_gpu_cross import HALF, Case, V, _hold, _step_case  # noqa: F401  (V: the fixture)
from vda_testutil import from_device

pytestmark = pytest.mark.gpu


def _run(V, c):
    d, o = c.dev, c.options()
    out, lse = V.cross_forward(d["q"], d["k"], d["v"], return_lse=True, **o)
    return out, lse, V.cross_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, **o)


GROUPS = {
    "33_few": dict(lq=[1], lk=[130], Hq=33, Hk=1, d=64),
    "33": dict(lq=[9, 9], lk=[70, 70], Hq=66, Hk=2, d=64, layout="heads", kv_layout="tokens"),
    "71_packed": dict(lq=[3, 0, 11], lk=[130, 5, 300], Hq=71, Hk=1, d=32, lead=2, tail=3, mask="holes"),
    "71_heads": dict(lq=[4, 6], lk=[65, 200], Hq=142, Hk=2, d=128, layout="heads", lead=1, tail=1),
    "128": dict(lq=[7], lk=[257], Hq=128, Hk=1, d=128, kv_layout="heads"),
    "1000": dict(lq=[3], lk=[90], Hq=1000, Hk=1, d=32, layout="heads", out_layout="tokens"),
    "1024": dict(lq=[1, 1], lk=[64, 64], Hq=1024, Hk=1, d=32, lens=[1, 64]),
    "1024_packed": dict(lq=[2, 1], lk=[700, 33], Hq=1024, Hk=1, d=64, layout="heads", mask="holes"),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", GROUPS)
def test_many_heads_to_a_key_head(V, name, dtype):
    print(name, dtype, flush=True)
    c = Case(dtype=dtype, **GROUPS[name])
    c.check(*_run(V, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H_q, H_k, t", [(33, 1, 1), (71, 1, 2), (142, 2, 1), (1024, 1, 1)])
def test_steps_of_many_heads_to_a_key_head(V, H_q, H_k, t, dtype):
    _step_case(V, n=3, t=t, m=4, S=150, Hq=H_q, Hk=H_k, d=64, dtype=dtype, kv_layout="tokens", lens=[150, 0, 31, 64], slots=[3, 0, 1])


@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_heads_past_32_bits_apart(V, layout):
    """Nine query heads of a key head, in the heads layout 268 MB apart, so that a tile's rows are not within 2^31 bytes of
    its first; in the tokens layout the same 2.4 GB, of tensors that are read whole.  All tokens but the last 70 ask nothing
    in particular (q = 0: the mean of v) and have no gradient."""
    import torch
    T, n, H, d, S = (1 << 20) + 37, 70, 9, 128, (90, 40)
    rng = np.random.default_rng(5)
    shape = (H, T, d) if layout == "heads" else (T, H, d)
    tail = (slice(None), slice(T - n, T)) if layout == "heads" else (slice(T - n, T),)
    as_tokens = (lambda x: x.transpose(0, 1)) if layout == "heads" else (lambda x: x)
    q, do = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    host = {}
    for name, x in (("q", q), ("do", do)):
        v = torch.from_numpy(rng.standard_normal((n, H, d))).bfloat16()
        x[tail] = as_tokens(v).cuda()
        host[name] = v.double().numpy()
    kv = [torch.from_numpy(rng.standard_normal((sum(S), 1, d))).bfloat16() for _ in range(2)]
    k, v = (x.cuda() for x in kv)
    o = dict(layout=layout, kv_layout="tokens", out_layout=layout,
             cu_q=torch.tensor([0, T - n, T], dtype=torch.int32, device="cuda"),
             cu_k=torch.tensor([0, S[0], sum(S)], dtype=torch.int32, device="cuda"))
    out, lse = V.cross_forward(q, k, v, return_lse=True, **o)
    dq, dk, dv = V.cross_backward(do, q, k, v, out, lse, **o)
    kh, vh = (x[S[0]:].double().numpy() for x in kv)
    a = (host["q"], kh, vh, np.ones(S[1], bool), d ** -0.5)
    want, bound = X.cross_sequence(*a, host["do"]), X.cross_bounds(*a, HALF["bf16"], host["do"])
    got = (from_device(as_tokens(out[tail]).contiguous()), from_device(lse[:, T - n:].t().contiguous()),
           from_device(as_tokens(dq[tail]).contiguous()), from_device(dk[S[0]:]), from_device(dv[S[0]:]))
    for g, w, b, name in zip(got, want, bound, ("out", "lse", "dq", "dk", "dv")):
        _hold(g, w, b, name)
    # The first sequence's rows: every head's first, one inside and its last.
    at = torch.tensor([0, (T - n) // 2, T - n - 1], device="cuda")
    some = from_device(as_tokens(out.index_select(1 if layout == "heads" else 0, at)).contiguous())
    k0, v0 = (x[:S[0]].double().numpy() for x in kv)
    a = (np.zeros((3, H, d)), k0, v0, np.ones(S[0], bool), d ** -0.5)
    _hold(some, X.cross_sequence(*a)[0], X.cross_bounds(*a, HALF["bf16"])[0], "mean")
    assert not dk[:S[0]].any() and not dv[:S[0]].any()
    assert not dq.index_select(1 if layout == "heads" else 0, at).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_largest_stride(V, dtype):
    """Rows almost 2^24 bytes apart, in slices of tensors of 2.5 GB: a tile of 128 states spans 2^31 bytes."""
    import torch
    c = Case(lq=[140], lk=[150], Hq=4, Hk=2, d=64, dtype=dtype, packed=True, mask="holes")
    es = 2 if dtype == "bf16" else 4
    wide = ((1 << 24) - 16) // es

    def slices(*tensors):
        """The [rows, H, d] tensors side by side in the rows of one wide buffer."""
        buf = torch.empty(tensors[0].shape[0] * wide, dtype=c.dt, device="cuda")
        got, at = [], wide - sum(t[0].numel() for t in tensors)
        for t in tensors:
            view = buf.as_strided(t.shape, (wide, c.d, 1), at)
            view.copy_(t)
            got.append(view)
            at += t[0].numel()
        return got

    d, o = c.dev, c.options()
    q, = slices(d["q"])
    k, v = slices(d["k"], d["v"])
    out, lse = V.cross_forward(q, k, v, return_lse=True, **o)
    dq, = slices(torch.full_like(d["q"], 3.0))
    dk, dv = slices(*(torch.full_like(d["k"], 3.0) for _ in range(2)))
    V.cross_backward(d["dout"], q, k, v, out, lse, outs=(dq, dk, dv), **o)
    c.check(out, lse, (dq, dk, dv))
