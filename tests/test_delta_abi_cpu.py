"""Host-side checks of the delta rule's and the rotary positions' entry points
(no GPU): invalid arguments are refused before anything is enqueued, and the
workspaces grow as documented."""
import ctypes

import pytest

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")

BIG = 1 << 36  # distinct, far-apart fake device addresses; validation never dereferences them
OK, NULL, SIZE, UNSUPPORTED, ALIGN, OVERLAP = 0, 1, 2, 3, 4, 5


def _problem(**kw):
    a = dict(T=200, n_seqs=2, cu_seqlens=None, H_k=2, H_v=4, d_k=64, d_v=128, layout=0, is_f32=0, scale=1.0)
    a.update(kw)
    return vda.VdaDeltaProblem(*a.values())


FORWARD = ("q", "k", "v", "g", "beta", "S_in", "out", "S_out", "work")
BACKWARD = ("dout", "q", "k", "v", "g", "beta", "S_in", "dS_out", "dq", "dk", "dv", "dg", "dbeta", "dS_in", "work")


def _call(names, fn, problem, **kw):
    args = {n: (i + 1) * BIG for i, n in enumerate(names)}
    args.update(kw)
    return fn(ctypes.byref(problem) if problem is not None else None, *args.values(), None)


def _forward(problem=None, **kw):
    return _call(FORWARD, vda.lib.vda_delta_forward, problem or _problem(), **kw)


def _backward(problem=None, **kw):
    return _call(BACKWARD, vda.lib.vda_delta_backward, problem or _problem(), **kw)


@pytest.mark.parametrize("fn,names", [(_forward, FORWARD), (_backward, BACKWARD)], ids=["forward", "backward"])
def test_delta_refusals(fn, names):
    optional = {"S_in", "S_out", "dS_out", "dS_in"}
    for n in names:
        if n not in optional:
            assert fn(**{n: None}) == NULL, n
    for bad, st in [(dict(T=0), SIZE), (dict(n_seqs=0), SIZE), (dict(n_seqs=3), SIZE), (dict(H_k=0), SIZE),
                    (dict(H_v=3), SIZE), (dict(H_v=0), SIZE), (dict(d_k=16), UNSUPPORTED), (dict(d_v=96), UNSUPPORTED),
                    (dict(d_k=256), UNSUPPORTED), (dict(layout=2), UNSUPPORTED), (dict(cu_seqlens=BIG + 2), ALIGN),
                    (dict(layout=1, H_v=1 << 20, H_k=1 << 20, T=2), SIZE), (dict(T=1 << 30, n_seqs=1, H_v=64), SIZE),
                    (dict(T=0x7fffffff, n_seqs=1), SIZE)]:
        assert fn(_problem(**bad)) == st, bad
    for i, n in enumerate(names):
        off = 2 if n in ("g", "beta", "dg", "dbeta") else 8
        assert fn(**{n: (i + 1) * BIG + off}) == ALIGN, n


def test_delta_overlaps():
    for n in ("q", "k", "v", "g", "beta", "S_in", "S_out", "work"):
        assert _forward(**{n: 7 * BIG}) == OVERLAP, n  # the output's place
    assert _forward(_problem(cu_seqlens=7 * BIG)) == OVERLAP
    assert _forward(S_out=6 * BIG) == OVERLAP  # the entering state's place: not in place
    for n in ("q", "k", "v", "g", "beta", "S_in", "dS_out", "dout", "dk", "dv", "dg", "dbeta", "dS_in", "work"):
        assert _backward(**{n: 9 * BIG}) == OVERLAP, n  # dq's place


def test_delta_workspace():
    fwd, bwd = vda.lib.vda_delta_forward_workspace, vda.lib.vda_delta_backward_workspace
    for bad in (None, _problem(T=0), _problem(d_k=16), _problem(H_v=3)):
        assert fwd(ctypes.byref(bad) if bad else None) == 0
        assert bwd(ctypes.byref(bad) if bad else None) == 0
    small, large = _problem(), _problem(T=20000)
    assert 0 < fwd(ctypes.byref(small)) < fwd(ctypes.byref(large)) < bwd(ctypes.byref(large))
    # The states at every chunk and their gradients are the backward pass's: 16 d_k d_v bytes a chunk and head.
    chunks = 2 * ((100 + 63) // 64) * 4
    assert bwd(ctypes.byref(small)) >= chunks * 8 * 64 * 128
    # Nothing past the work buffer's own size counts as it.
    n = fwd(ctypes.byref(small))
    assert _forward(work=7 * BIG - n + 16) == OVERLAP


STEP = ("q", "k", "v", "g", "beta", "n", "tokens", "H_k", "H_v", "d_k", "d_v", "is_f32", "scale", "slots", "n_slots",
        "state", "out")


def _step(**kw):
    a = dict(q=BIG, k=2 * BIG, v=3 * BIG, g=4 * BIG, beta=5 * BIG, n=3, tokens=2, H_k=2, H_v=4, d_k=64, d_v=32,
             is_f32=0, scale=1.0, slots=6 * BIG, n_slots=8, state=7 * BIG, out=8 * BIG)
    a.update(kw)
    return vda.lib.vda_delta_step(*(a[n] for n in STEP), None)


def test_step_refusals():
    for n in ("q", "k", "v", "g", "beta", "state", "out"):
        assert _step(**{n: None}) == NULL, n
    for bad, st in [(dict(n=0), SIZE), (dict(tokens=0), SIZE), (dict(n_slots=0), SIZE), (dict(H_v=5), SIZE),
                    (dict(slots=None, n=9), SIZE), (dict(d_k=48), UNSUPPORTED), (dict(d_v=16), UNSUPPORTED),
                    (dict(n=1 << 24, H_v=64), SIZE), (dict(n=1 << 20, tokens=1 << 12), SIZE),
                    (dict(q=BIG + 8), ALIGN), (dict(state=7 * BIG + 4), ALIGN), (dict(slots=6 * BIG + 2), ALIGN),
                    (dict(out=7 * BIG + 4096), OVERLAP), (dict(out=3 * BIG), OVERLAP), (dict(slots=8 * BIG), OVERLAP),
                    (dict(g=7 * BIG + 64), OVERLAP)]:
        assert _step(**bad) == st, bad


def _rope(backward=False, x=BIG, dout=2 * BIG, inv_freq=3 * BIG, positions=4 * BIG, B=2, L=10, H=3, d=64, is_f32=0,
          out=5 * BIG, **opts):
    o = dict(pairs_t=8, pairs_h=8, pairs_w=16, interleaved=1, l2=1, layout=0, grid_h=0, grid_w=0, frame_offset=0,
             x_row_stride=0, dx_row_stride=0)
    o.update(opts)
    ro = vda.VdaRopeOptions(*o.values())
    if backward:
        return vda.lib.vda_rope_backward(dout, x, inv_freq, positions, B, L, H, d, ctypes.byref(ro), is_f32, out, None)
    return vda.lib.vda_rope(x, inv_freq, positions, B, L, H, d, ctypes.byref(ro), is_f32, out, None)


@pytest.mark.parametrize("backward", [False, True])
def test_rope_refusals(backward):
    grid = dict(positions=None, grid_h=2, grid_w=5)
    for bad, st in [(dict(inv_freq=None), NULL), (dict(out=None), NULL), (dict(x=None), NULL), (dict(B=0), SIZE),
                    (dict(L=0), SIZE), (dict(H=0), SIZE), (dict(d=48), UNSUPPORTED), (dict(d=256), UNSUPPORTED),
                    (dict(pairs_t=-8), SIZE), (dict(pairs_t=0, pairs_h=0, pairs_w=0), SIZE), (dict(pairs_t=16), SIZE),
                    (dict(pairs_t=4), UNSUPPORTED), (dict(layout=5), UNSUPPORTED), (dict(**grid, frame_offset=-1), SIZE),
                    (dict(positions=None), SIZE), (dict(**grid, frame_offset=0x7fffffff), SIZE),
                    (dict(x_row_stride=100), SIZE), (dict(x_row_stride=196), ALIGN), (dict(x=BIG + 8), ALIGN),
                    (dict(out=5 * BIG + 8), ALIGN), (dict(inv_freq=3 * BIG + 2), ALIGN), (dict(out=BIG), OVERLAP),
                    (dict(out=3 * BIG), OVERLAP), (dict(out=4 * BIG), OVERLAP), (dict(H=1 << 25), SIZE),
                    (dict(B=1 << 16, L=1 << 12), SIZE)]:
        assert _rope(backward, **bad) == st, bad
    if backward:
        assert _rope(True, dout=None) == NULL
        assert _rope(True, out=2 * BIG) == OVERLAP
        assert _rope(True, dx_row_stride=100) == SIZE
        assert _rope(True, dx_row_stride=196) == ALIGN


def test_binding_refuses_cpu_tensors():
    import torch
    q = torch.zeros(1, 4, 32)
    with pytest.raises(ValueError):
        vda.delta_forward(q, q, q, q[..., 0], q[..., 0])
    with pytest.raises(ValueError):
        vda.rope(torch.zeros(1, 4, 32), torch.zeros(8), (8, 0, 0), 1, grid=(2, 2))
    with pytest.raises(ValueError):
        vda.delta_step(*(torch.zeros(1, 1, 1, 32),) * 3, torch.zeros(1, 1, 1), torch.zeros(1, 1, 1),
                       torch.zeros(1, 1, 32, 32))


def test_most_sequences():
    """The join has a workgroup for 16 rows of every state, of a count that is rounded up to eight: below 2^32 threads."""
    need = lambda **kw: vda.lib.vda_delta_forward_workspace(  # noqa: E731
        ctypes.byref(_problem(T=64, cu_seqlens=BIG, H_k=1, H_v=1, **kw)))
    assert need(n_seqs=(1 << 21) - 8, d_v=128) > 0
    assert need(n_seqs=(1 << 21) - 1, d_v=128) == 0
    assert need(n_seqs=(1 << 21) - 1, d_v=64) > 0
    assert need(n_seqs=1 << 22, d_v=32) == 0
