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
