"""GPU test of the rotary gradient through the L2 map where it cancels: gradients
along the token itself, of which dy - xh (xh . dy) leaves little.

Tolerance: the result is rounded once to the storage type (bf16: 2^-8 of it);
what is subtracted is fp32 of dy's size, about 24 roundings of 2^-24 (as in
test_gpu_rope.py) of |dy| / n, n the token's length."""
import numpy as np
import pytest

import oracle.delta_oracle as D
from vda_testutil import from_device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("d,axes", [(16, (2, 3, 3)), (64, (8, 12, 12)), (128, (8, 12, 12))])
def test_gradients_along_the_token(d, axes, interleaved, dtype):
    import torch
    from paper_2609_20744_amd import vda as V
    rng = np.random.default_rng(d)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    B, H, gh, gw, F = 1, 3, 3, 4, 5
    L = gh * gw * F
    pos = D.grid_positions(L, gh, gw, 7)
    f = torch.from_numpy(np.concatenate([100.0 ** (-np.arange(a) / a) for a in axes])).float()
    x = torch.from_numpy(rng.standard_normal((B, L, H * d)) * 2.0 ** rng.integers(-6, 7, (B, L, 1))).to(dt)
    heads = [x[0, :, h * d:(h + 1) * d].double().numpy() for h in range(H)]
    along = np.stack([D.rope_head(z, pos, f.numpy(), axes, interleaved, False) for z in heads])
    dy = torch.from_numpy(along).to(dt)
    got = from_device(V.rope_backward(dy.cuda(), f.cuda(), axes, H, x=x.cuda(), grid=(gh, gw), frame_offset=7, l2=True,
                                      interleaved=interleaved))[0]
    for h in range(H):
        want = D.rope_head_backward(dy[h].double().numpy(), heads[h], pos, f.numpy(), axes, interleaved, True)
        n = np.sqrt((heads[h] ** 2).sum(-1) + 1e-6)
        size = np.linalg.norm(dy[h].double().numpy(), axis=-1) / n
        err = np.linalg.norm(got[:, h * d:(h + 1) * d] - want, axis=-1)
        bound = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.linalg.norm(want, axis=-1) + 24 * 2.0 ** -24 * size
        assert (err <= bound).all(), float((err / bound).max())
        # What is left is far below what was there.
        assert (np.linalg.norm(want, axis=-1) <= 2.0 ** -7 * size).all()
