"""Plans and refusals of the cross attention and the recurrence at the largest sizes
that their entry points take (no GPU: workspace queries, and calls that are refused
before anything is enqueued)."""
import ctypes

import pytest

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")

BIG = 1 << 44  # distinct, far-apart fake device addresses; validation never dereferences them
OK, NULL, SIZE, UNSUPPORTED, ALIGN, OVERLAP = 0, 1, 2, 3, 4, 5
TOKENS = 1


def _cross(T, S, n_seqs=1, H_q=1, H_k=1, d=32, is_f32=0, cu_q=None, cu_k=None):
    return vda.VdaCrossProblem(T, S, n_seqs, cu_q, cu_k, None, None, H_q, H_k, d, TOKENS, TOKENS, TOKENS, 0, 0, 0, 0, 0, 0,
                               is_f32, 1.0)


def _backward(problem, **kw):
    """Refused for dq's place at the latest, which is that of q."""
    names = ("dout", "q", "k", "v", "out", "lse", "dq", "dk", "dv", "work")
    args = {n: (i + 1) * BIG for i, n in enumerate(names)}
    args["dq"] = args["q"]
    args.update(kw)
    return vda.lib.vda_cross_backward(ctypes.byref(problem), *args.values(), None)


@pytest.mark.parametrize("is_f32", [0, 1])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("T,S,H", [
    (3 << 20, 1 << 23, 16),                # rows * groups / (3 * 256) is 2^32
    (768 << 11, (1 << 28) + 128, 1),       # a little more than 2^32
    (1 << 26, 1 << 26, 1),                 # more than 2^31, below 2^32
    ((1 << 29) - 512, (1 << 29) - 512, 1),  # close to the most that the checks let through
    ((1 << 25) - 128, (1 << 25) - 128, 16),
])
def test_cross_rows_of_large_problems_are_one_range(T, S, H, packed, is_f32):
    """Where the states' tiles alone are many times the device's compute units, the rows are one range: the workspace has D
    and lse of every row and a count for every state, and no parts."""
    p = _cross(T, S, H_q=H, H_k=H, is_f32=is_f32, cu_q=30 * BIG if packed else None, cu_k=31 * BIG if packed else None)
    up = lambda x: (x + 255) // 256 * 256
    assert vda.lib.vda_cross_backward_workspace(ctypes.byref(p)) == up(T * H * 8) + up(S * 4)
    assert _backward(p) == OVERLAP


@pytest.mark.parametrize("is_f32,threads", [(0, 512), (1, 256)])
@pytest.mark.parametrize("packed", [False, True])
def test_cross_backward_workgroups_fit_a_launch(packed, is_f32, threads):
    """The gradients of k and v take a workgroup for 128 states, of 512 threads in bf16 storage; a launch holds 2^32 - 1."""
    most = (2 ** 32 - 1) // threads
    for n, st in (((most - 16) // 2, OVERLAP), (most + 16, SIZE), (9 << 20, SIZE if is_f32 == 0 else OVERLAP), (most * 2, SIZE)):
        p = _cross(n, n, n_seqs=n, is_f32=is_f32, cu_q=30 * BIG if packed else None, cu_k=31 * BIG if packed else None)
        assert _backward(p) == st, n
        assert (vda.lib.vda_cross_backward_workspace(ctypes.byref(p)) > 0) == (st == OVERLAP)
    p = _cross(9 << 20, 9 << 20, n_seqs=9 << 20)
    assert vda.lib.vda_cross_forward(ctypes.byref(p), BIG, 2 * BIG, 3 * BIG, BIG, None, None, None) == OVERLAP  # allowed: 256 threads


def _recur(T, C, n_seqs=1, cu=None):
    return vda.VdaRecurProblem(T, n_seqs, cu, C, 1, 0, 0, 0, 0, 0, 0)


def _recur_backward(problem):
    """Refused for dx's place at the latest, which is that of x."""
    x = 2 * BIG
    return vda.lib.vda_recur_backward(ctypes.byref(problem), BIG, x, 3 * BIG, None, None, x, 4 * BIG, None, 5 * BIG, None)


def test_recur_channels_fit_a_launch():
    """What enters each tile is found by a workgroup for 64 channels of a sequence, the channels along the grid's second
    dimension, of 65535 at most; a sequence of one tile (64 tokens) does without."""
    most = 64 * 65535
    for T, C, n, cu, st in ((65, most, 1, None, OVERLAP), (65, most + 8, 1, None, SIZE), (65, most + 64, 1, None, SIZE),
                            (65, 128 * 65535, 1, None, SIZE), (64, most + 64, 1, None, OVERLAP), (128, most + 64, 2, None, OVERLAP),
                            (128, most + 64, 2, 9 * BIG, SIZE), (130, most + 64, 2, None, SIZE), (64, 128 * 65535, 1, None, OVERLAP)):
        p = _recur(T, C, n, cu)
        assert _recur_backward(p) == st, (T, C, n, cu)
        assert (vda.lib.vda_recur_backward_workspace(ctypes.byref(p)) > 0) == (st == OVERLAP and C <= most)
    p = _recur(1000, 128 * 65535)
    assert vda.lib.vda_recur_forward(ctypes.byref(p), BIG, 2 * BIG, None, BIG, None, 5 * BIG, None) == OVERLAP
