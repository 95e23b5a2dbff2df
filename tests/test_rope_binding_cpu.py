"""Host-side checks of the rotary positions' binding (no GPU): what the C call
cannot see, because its arguments are 32-bit, is refused before it."""
import pytest
import torch

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")


@pytest.mark.parametrize("H", [0, -1, -4])
def test_head_counts_below_one(H):
    with pytest.raises(ValueError):
        vda._token_rows(torch.zeros(1, 4, 32), "x", H)


@pytest.mark.gpu
@pytest.mark.parametrize("H", [0, -2])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_head_counts_below_one_through_the_calls(H, layout):
    x, f = torch.zeros(2, 4, 32, device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(ValueError):
        vda.rope(x, f, (8, 0, 0), H, grid=(2, 2), layout=layout)
    with pytest.raises(ValueError):
        vda.rope_backward(x, f, (8, 0, 0), H, grid=(2, 2), layout=layout)
