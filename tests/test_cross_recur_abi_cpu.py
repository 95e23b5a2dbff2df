"""Host-side checks of the cross attention's and the recurrence's entry points (no
GPU): invalid arguments are refused before anything is enqueued, and the
workspaces grow as documented."""
import ctypes

import pytest

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")

BIG = 1 << 36  # distinct, far-apart fake device addresses; validation never dereferences them
OK, NULL, SIZE, UNSUPPORTED, ALIGN, OVERLAP = 0, 1, 2, 3, 4, 5
HEADS, TOKENS = 0, 1


def _cross(**kw):
    a = dict(T=200, S=60, n_seqs=2, cu_q=None, cu_k=None, k_lens=20 * BIG, k_mask=21 * BIG, H_q=8, H_k=2, d=64, layout=TOKENS,
             kv_layout=TOKENS, out_layout=TOKENS, q_row_stride=0, k_row_stride=0, v_row_stride=0, dq_row_stride=0,
             dk_row_stride=0, dv_row_stride=0, is_f32=0, scale=1.0)
    a.update(kw)
    return vda.VdaCrossProblem(*a.values())


FORWARD = ("q", "k", "v", "out", "lse", "work")
BACKWARD = ("dout", "q", "k", "v", "out", "lse", "dq", "dk", "dv", "work")


def _call(names, fn, problem, **kw):
    args = {n: (i + 1) * BIG for i, n in enumerate(names)}
    args.update(kw)
    return fn(ctypes.byref(problem), *args.values(), None)


def _forward(problem=None, **kw):
    return _call(FORWARD, vda.lib.vda_cross_forward, problem or _cross(), **kw)


def _backward(problem=None, **kw):
    return _call(BACKWARD, vda.lib.vda_cross_backward, problem or _cross(), **kw)


def _step(problem=None, slots=9 * BIG, n_slots=2, **kw):
    a = {n: (i + 1) * BIG for i, n in enumerate(("q", "k", "v", "out", "work"))}
    a.update(kw)
    return vda.lib.vda_cross_step(ctypes.byref(problem or _cross()), a["q"], a["k"], a["v"], slots, n_slots, a["out"], a["work"],
                                  None)


BAD = [(dict(T=0), SIZE), (dict(S=0), SIZE), (dict(n_seqs=0), SIZE), (dict(n_seqs=3), SIZE), (dict(H_k=0), SIZE),
       (dict(H_q=0), SIZE), (dict(H_q=5), SIZE), (dict(d=16), UNSUPPORTED), (dict(d=96), UNSUPPORTED),
       (dict(d=256), UNSUPPORTED), (dict(layout=2), UNSUPPORTED), (dict(kv_layout=-1), UNSUPPORTED),
       (dict(out_layout=7), UNSUPPORTED), (dict(H_q=4096, H_k=1), UNSUPPORTED), (dict(k_lens=BIG + 2), ALIGN),
       (dict(q_row_stride=511), SIZE), (dict(k_row_stride=127), SIZE), (dict(q_row_stride=516), ALIGN),
       (dict(v_row_stride=132), ALIGN), (dict(k_row_stride=1 << 23), SIZE), (dict(q_row_stride=-512), SIZE),
       (dict(layout=HEADS, q_row_stride=512), UNSUPPORTED), (dict(kv_layout=HEADS, k_row_stride=512), UNSUPPORTED),
       (dict(T=0x7fffffff, n_seqs=1, H_q=2), SIZE), (dict(S=0x7fffffff, n_seqs=1), SIZE),
       (dict(T=1 << 30, n_seqs=1, H_q=4), SIZE), (dict(H_q=1 << 18, H_k=1 << 18), SIZE)]


@pytest.mark.parametrize("fn", [_forward, _backward, _step], ids=["forward", "backward", "step"])
def test_cross_refusals(fn):
    for bad, st in BAD:
        assert fn(_cross(**bad)) == st, bad


def test_cross_null_and_alignment():
    for fn, names in ((_forward, FORWARD), (_backward, BACKWARD)):
        for i, n in enumerate(names):
            if fn is _backward or n in ("q", "k", "v", "out"):
                assert fn(**{n: None}) == NULL, n
            assert fn(_cross(S=6000, T=2), **{n: (i + 1) * BIG + (2 if n == "lse" else 8)}) == ALIGN, n
    assert _forward(_cross(S=6000, T=2), work=None) == NULL  # the states are shared out: the parts need room
    for n in ("q", "k", "v", "out"):
        assert _step(**{n: None}) == NULL
        assert _step(**{n: 50 * BIG + 8}) == ALIGN
    assert _step(slots=BIG // 2 + 2) == ALIGN
    assert _step(n_slots=0) == SIZE
    assert _step(n_slots=7) == SIZE  # 60 states of 7 slots
    assert _step(slots=None, n_slots=1) == SIZE  # two sequences, one slot
    assert _step(_cross(cu_q=BIG)) == SIZE
    assert _step(_cross(cu_k=BIG)) == SIZE
    assert vda.lib.vda_cross_forward(None, BIG, BIG, BIG, BIG, None, None, None) == NULL


def test_cross_overlaps():
    long = dict(S=6000, T=2)
    for n in ("q", "k", "v", "lse", "work"):
        assert _forward(_cross(**long), **{n: 4 * BIG}) == OVERLAP, n  # the output's place
    for f in ("cu_q", "cu_k", "k_lens", "k_mask"):
        assert _forward(_cross(**{f: 4 * BIG + 64})) == OVERLAP, f
        assert _backward(_cross(**{f: 7 * BIG + 64})) == OVERLAP, f
    for n in ("dout", "q", "k", "v", "out", "lse", "dk", "dv", "work"):
        assert _backward(**{n: 7 * BIG}) == OVERLAP, n  # dq's place
    assert _step(slots=4 * BIG) == OVERLAP
    # dk and dv as slices of one gradient: apart in every row, or not.
    row = 2 * 64 * 2
    fused = _cross(dk_row_stride=256, dv_row_stride=256)
    assert _backward(fused, dk=8 * BIG, dv=8 * BIG + row // 2) == OVERLAP
    assert _backward(_cross(dk_row_stride=256, dv_row_stride=512), dk=8 * BIG, dv=8 * BIG + row) == OVERLAP
    assert _backward(fused, dk=8 * BIG, dv=8 * BIG + row, q=8 * BIG + 64) == OVERLAP
    assert _backward(fused, dk=8 * BIG, dv=8 * BIG + row, work=8 * BIG + row) == OVERLAP


def test_cross_workspace():
    f, b, s = (getattr(vda.lib, f"vda_cross_{n}_workspace") for n in ("forward", "backward", "step"))
    for bad in (None, _cross(T=0), _cross(d=48), _cross(H_q=3)):
        p = ctypes.byref(bad) if bad is not None else None
        assert f(p) == b(p) == s(p, 2) == 0
    assert s(ctypes.byref(_cross()), 0) == 0
    many = _cross(T=1 << 16, S=2 * 512, H_q=16, H_k=16)
    assert f(ctypes.byref(many)) == 0  # rows enough: nothing is shared out
    assert b(ctypes.byref(many)) >= (1 << 16) * 16 * 8
    few = _cross(T=2, S=2 * 40000)
    n = f(ctypes.byref(few))
    assert n >= 2 * 2 * 8 * 64 * 4
    assert _forward(few, work=4 * BIG - n + 16) == OVERLAP


def _recur(**kw):
    a = dict(T=400, n_seqs=2, cu_seqlens=None, C=64, gate=1, reverse=0, x_row_stride=0, g_row_stride=0, dx_row_stride=0,
             dg_row_stride=0, is_f32=0)
    a.update(kw)
    return vda.VdaRecurProblem(*a.values())


R_FORWARD = ("x", "g", "S_in", "out", "S_out", "work")
R_BACKWARD = ("dout", "x", "g", "S_in", "dS_out", "dx", "dg", "dS_in", "work")


def _r_forward(problem=None, **kw):
    return _call(R_FORWARD, vda.lib.vda_recur_forward, problem or _recur(), **kw)


def _r_backward(problem=None, **kw):
    return _call(R_BACKWARD, vda.lib.vda_recur_backward, problem or _recur(), **kw)


@pytest.mark.parametrize("fn,names", [(_r_forward, R_FORWARD), (_r_backward, R_BACKWARD)], ids=["forward", "backward"])
def test_recur_refusals(fn, names):
    optional = {"S_in", "S_out", "dS_out", "dS_in"}
    for i, n in enumerate(names):
        if n not in optional:
            assert fn(**{n: None}) == NULL, n
        assert fn(**{n: (i + 1) * BIG + 8}) == ALIGN, n
    for bad, st in [(dict(T=0), SIZE), (dict(n_seqs=0), SIZE), (dict(n_seqs=3), SIZE), (dict(C=0), SIZE),
                    (dict(C=12), UNSUPPORTED), (dict(gate=3), UNSUPPORTED), (dict(gate=-1), UNSUPPORTED),
                    (dict(cu_seqlens=BIG + 2), ALIGN), (dict(x_row_stride=56), SIZE), (dict(g_row_stride=68), ALIGN),
                    (dict(x_row_stride=-64), SIZE), (dict(T=0x7fffffff, n_seqs=1), SIZE),
                    (dict(T=1 << 24, n_seqs=1 << 24), SIZE), (dict(C=128 * 65536), SIZE)]:
        assert fn(_recur(**bad)) == st, bad
    place = {n: (i + 1) * BIG for i, n in enumerate(names)}
    target = "out" if fn is _r_forward else "dx"
    for n in names:
        if n != target:
            assert fn(**{n: place[target]}) == OVERLAP, n
    assert fn(_recur(cu_seqlens=place[target] + 64)) == OVERLAP
    if fn is _r_backward:
        fused = dict(dx_row_stride=128, dg_row_stride=128)
        assert fn(_recur(**fused), dg=place["dx"] + 64) == OVERLAP
        assert fn(_recur(**fused, gate=0), dg=place["dx"] + 128) == OVERLAP  # fp32 beside bf16
        assert fn(_recur(**fused), dg=place["dx"] + 128, x=place["dx"] + 256) == OVERLAP
        assert fn(_recur(dx_row_stride=68)) == ALIGN and fn(_recur(dg_row_stride=56)) == SIZE


def test_recur_workspace():
    f, b = vda.lib.vda_recur_forward_workspace, vda.lib.vda_recur_backward_workspace
    for bad in (None, _recur(T=0), _recur(C=12), _recur(gate=5)):
        p = ctypes.byref(bad) if bad is not None else None
        assert f(p) == b(p) == 0
    assert f(ctypes.byref(_recur(T=16))) == 0  # short sequences leave nothing for others
    long = _recur(T=100000)
    assert 0 < f(ctypes.byref(long)) < b(ctypes.byref(long)) < 100000 * 64 * 4
    n = f(ctypes.byref(long))
    assert _r_forward(long, work=4 * BIG - n + 16) == OVERLAP
    assert _r_forward(long, work=None) == NULL


def test_recur_step_refusals():
    def step(**kw):
        a = dict(x=BIG, g=2 * BIG, n=3, tokens=2, C=64, gate=0, is_f32=0, slots=3 * BIG, n_slots=8, state=4 * BIG, out=5 * BIG)
        a.update(kw)
        return vda.lib.vda_recur_step(*a.values(), None)
    for n in ("x", "g", "state", "out"):
        assert step(**{n: None}) == NULL, n
    for bad, st in [(dict(n=0), SIZE), (dict(tokens=0), SIZE), (dict(n_slots=0), SIZE), (dict(C=0), SIZE),
                    (dict(C=20), UNSUPPORTED), (dict(gate=9), UNSUPPORTED), (dict(slots=None, n=9), SIZE),
                    (dict(n=1 << 30, C=1 << 10), SIZE), (dict(n=1 << 20, tokens=1 << 12), SIZE), (dict(x=BIG + 8), ALIGN),
                    (dict(state=4 * BIG + 4), ALIGN), (dict(slots=3 * BIG + 2), ALIGN), (dict(out=4 * BIG + 512), OVERLAP),
                    (dict(out=BIG), OVERLAP), (dict(slots=5 * BIG), OVERLAP), (dict(g=4 * BIG + 64), OVERLAP)]:
        assert step(**bad) == st, bad


def test_binding_refuses_cpu_tensors():
    import torch
    q = torch.zeros(1, 4, 2, 32)
    with pytest.raises(ValueError):
        vda.cross_forward(q, q, q)
    with pytest.raises(ValueError):
        vda.cross_step(q, q, q)
    with pytest.raises(ValueError):
        vda.recur_forward(torch.zeros(4, 8), torch.zeros(4, 8))
    with pytest.raises(ValueError):
        vda.recur_step(torch.zeros(1, 1, 8), torch.zeros(1, 1, 8), torch.zeros(1, 8))


def test_row_strides():
    """The binding takes slices of fused tensors and refuses tensors whose rows are not at one stride."""
    import torch
    rows = vda._row_stride
    fused = torch.zeros(2, 5, 3, 4, 8)  # [B, L, 3, H, d]
    assert rows(fused[:, :, 1], "t", 2) == 3 * 32
    assert rows(torch.zeros(2, 5, 4, 8), "t", 2) == 0
    assert rows(fused[:1, :1, 1], "t", 2) == 0  # one row
    assert rows(torch.zeros(2, 5, 48)[..., 8:24], "t", 1) == 48
    assert rows(torch.zeros(6, 48)[:, 16:32], "t", 1) == 48
    assert rows(torch.zeros(3, 6, 16)[:, ::2], "t", 1) == 32
    for bad, inner in ((torch.zeros(2, 4, 5, 8).transpose(1, 2), 2), (torch.zeros(5, 16)[:, ::2], 1),
                       (torch.zeros(3, 6, 16)[:, :4], 1), (torch.zeros(4, 16).t(), 1),
                       (torch.zeros(1, 16).expand(5, 16), 1), (torch.zeros(40).as_strided((5, 16), (6, 1)), 1)):
        with pytest.raises(ValueError):
            rows(bad, "t", inner)
