"""Checks of the rotary positions' Python binding: calls that the C entry point
does not see as they are, because its arguments are 32-bit, are refused before it."""
import pytest
import torch

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")


@pytest.mark.parametrize("H", [0, -1, -4])
def test_head_counts_below_one(H):
    with pytest.raises(ValueError):
        vda._token_rows(torch.zeros(1, 4, 32), "x", H)


def _args(**kw):
    a = dict(axes=(8, 0, 0), H=2, B=1, L=4, d=32, positions=None, grid=(2, 2), frame_offset=0)
    a.update(kw)
    inv_freq = torch.ones(8) if sum(a["axes"]) == 8 else torch.ones(16)
    return vda._rope_args(inv_freq, a["axes"], a["H"], a["B"], a["L"], a["d"], a["positions"], a["grid"],
                          a["frame_offset"], True, False, "heads", torch.device("cpu"))


@pytest.mark.parametrize("kw", [dict(frame_offset=(1 << 32) + 5), dict(frame_offset=-(1 << 32)),
                                dict(grid=((1 << 32) + 2, 2)), dict(grid=(2, (1 << 33) + 2)),
                                dict(axes=((1 << 32) + 8, -(1 << 32), 8)), dict(L=(1 << 32) + 4),
                                dict(B=(1 << 32) + 1), dict(H=(1 << 32) + 2)], ids=str)
def test_integers_past_32_bits(kw):
    """Not taken modulo 2^32, in which each of these is a sound call."""
    _args()
    with pytest.raises(ValueError):
        _args(**kw)


def test_rows_past_32_bits_apart():
    far = torch.empty_strided((1, 2, 32), (1, (1 << 32) + 64, 1), device="meta")
    with pytest.raises(ValueError):
        vda._token_rows(far, "x", 1)
    assert vda._token_rows(torch.empty_strided((1, 2, 32), (1, (1 << 31) - 8, 1), device="meta"), "x", 1) == (1 << 31) - 8


@pytest.mark.gpu
@pytest.mark.parametrize("H", [0, -2])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_head_counts_below_one_through_the_calls(H, layout):
    x, f = torch.zeros(2, 4, 32, device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(ValueError):
        vda.rope(x, f, (8, 0, 0), H, grid=(2, 2), layout=layout)
    with pytest.raises(ValueError):
        vda.rope_backward(x, f, (8, 0, 0), H, grid=(2, 2), layout=layout)


def test_input_that_is_not_read_is_not_checked():
    """Without l2 the gradient does not read x.  (Every call below is refused for its output's place, after the checks
    of alignment and strides, so nothing is launched on the made-up addresses.)"""
    import ctypes
    big = 1 << 36

    def call(x, stride, l2):
        o = vda.VdaRopeOptions(8, 8, 16, 1, l2, 0, 1, 1, 0, stride, 0)
        return vda.lib.vda_rope_backward(2 * big, x, 3 * big, 4 * big, 2, 10, 3, 64, ctypes.byref(o), 0, 2 * big, None)

    overlap, align, size = 5, 4, 2
    assert call(None, 0, 0) == overlap
    assert call(big + 8, 0, 0) == overlap and call(big + 8, 0, 1) == align
    assert call(big, 100, 0) == overlap and call(big, 100, 1) == size
    assert call(big, 196, 0) == overlap and call(big, 196, 1) == align


@pytest.mark.gpu
def test_input_that_is_not_read_may_have_any_form():
    f = torch.rand(16, device="cuda")
    dy = torch.randn(2, 6, 2 * 32, device="cuda")
    kw = dict(grid=(2, 3), layout="tokens")
    want = vda.rope_backward(dy, f, (4, 6, 6), 2, **kw)
    x = torch.zeros(2, 12, 2 * 32 + 1, device="cuda")[:, ::2, 1:]
    assert torch.equal(vda.rope_backward(dy, f, (4, 6, 6), 2, x=x, **kw), want)
    with pytest.raises(ValueError):
        vda.rope_backward(dy, f, (4, 6, 6), 2, x=x, l2=True, **kw)
