"""GPU parity of the rotary positions (rope, rope_backward) against the fp64
oracle.

Tolerances, of the largest output of a head: bf16 rounds each output once, by
at most 2^-8 of its value; fp32 arithmetic takes about 12 roundings of 2^-24
(the sums of the L2 map are of d squares, d / 16 at a time in a lane), the
angle's own error is 2^-24 of half a turn (pi 2^-24) and the sine's and
cosine's 2 * 2^-24."""
import numpy as np
import pytest

import oracle.delta_oracle as D
from vda_testutil import from_device

pytestmark = pytest.mark.gpu
TOL = {"bf16": 2.0 ** -8 + 24 * 2.0 ** -24, "f32": 24 * 2.0 ** -24}


@pytest.fixture(scope="module")
def V():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2609_20744_amd import vda
    return vda


CASES = [  # B, L, H, d, axes, grid, offset
    (1, 1, 1, 16, (8, 0, 0), (1, 1), 0),
    (1, 1, 5, 128, (16, 24, 24), None, 0),
    (2, 7, 3, 32, (4, 6, 6), None, 1 << 20),
    (1, 3 * 20 + 1, 2, 64, (8, 12, 12), (4, 5), 9),
    (3, 13, 1, 128, (8, 12, 12), None, -300),   # half of the channels, negative positions
    (2, 2 * 21, 4, 64, (0, 1, 7), (3, 7), 1 << 30),
    (1, 130, 24, 128, (64, 0, 0), (1, 1), 5),
    (2, 5, 2, 16, (2, 3, 3), None, (1 << 31) - 1 - 40),
]


def _case(B, L, H, d, axes, grid, offset, dtype, seed=0):
    import torch
    rng = np.random.default_rng(seed + L + d)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy(rng.standard_normal((B, L, H * d))).to(dt)
    dy = torch.from_numpy(rng.standard_normal((B, H, L, d))).to(dt)
    if B * L > 1:
        x[0, 0, :d] = 0.0  # a token without length
    f = torch.from_numpy(np.concatenate([10000.0 ** (-np.arange(a) / max(a, 1)) for a in axes])).float()
    if grid is None:
        pos = rng.integers(0, 40, (B, L, 3)) + offset
    else:
        pos = np.broadcast_to(D.grid_positions(L, *grid, offset), (B, L, 3))
    return x, dy, f, pos


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("interleaved,l2", [(True, False), (False, True), (True, True), (False, False)])
@pytest.mark.parametrize("B,L,H,d,axes,grid,offset", CASES, ids=[f"B{c[0]}_L{c[1]}_H{c[2]}_d{c[3]}" for c in CASES])
def test_rope_and_gradient(V, B, L, H, d, axes, grid, offset, interleaved, l2, layout, dtype):
    import torch
    x, dy, f, pos = _case(B, L, H, d, axes, grid, offset, dtype)
    kw = dict(interleaved=interleaved, l2=l2, layout=layout)
    if grid is None:
        kw["positions"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
    else:
        kw.update(grid=grid, frame_offset=offset)
    y = V.rope(x.cuda(), f.cuda(), axes, H, **kw)
    dout = (dy.flatten(0, 1) if layout == "heads" else dy.transpose(1, 2).flatten(2)).contiguous().cuda()
    dx = V.rope_backward(dout, f.cuda(), axes, H, x=x.cuda() if l2 else None, **kw)
    y, dx = from_device(y), from_device(dx)
    y = y.reshape(B, H, L, d) if layout == "heads" else y.reshape(B, L, H, d).transpose(0, 2, 1, 3)
    dx = dx.reshape(B, L, H, d).transpose(0, 2, 1, 3)
    for b in range(B):
        for h in range(H):
            xh = x[b, :, h * d:(h + 1) * d].double().numpy()
            ref = D.rope_head(xh, pos[b], f.numpy(), axes, interleaved, l2)
            ref_dx = D.rope_head_backward(dy[b, h].double().numpy(), xh, pos[b], f.numpy(), axes, interleaved, l2)
            # Of each token: a token without length has a gradient of its own size.
            for got, want in ((y[b, h], ref), (dx[b, h], ref_dx)):
                err = np.abs(got - want).max(-1)
                # dy - xh (xh . dy) can cancel: its roundings are of dy's size.
                size = np.abs(want).max(-1) + (np.abs(dy[b, h].double().numpy()).max(-1) / np.sqrt(
                    (xh ** 2).sum(-1) + 1e-6) * 8 * 2.0 ** -8 if l2 and got is dx[b, h] else 0)
                assert (err <= TOL[dtype] * np.maximum(size, 1e-30)).all(), (b, h, float((err / np.maximum(size, 1e-30)).max()))


def test_far_positions_keep_their_angle(V):
    """At positions of 2^31 - 1 an angle formed in fp32 would be off by tens of turns."""
    import torch
    x = torch.zeros(1, 1, 16, device="cuda")
    x[..., 0::2] = 1.0
    f = torch.linspace(0.3, 1.0, 8, device="cuda")
    p = torch.full((1, 1, 3), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    y = from_device(V.rope(x, f, (8, 0, 0), 1, positions=p, layout="tokens"))[0, 0]
    a = np.float64(2 ** 31 - 1) * f.double().cpu().numpy()
    # The product in 64 bits: 2^-53 of 2^31 / (2 pi) turns.
    assert np.abs(y[0::2] - np.cos(a)).max() <= 24 * 2.0 ** -24
    assert np.abs(y[1::2] - np.sin(a)).max() <= 24 * 2.0 ** -24


def test_slices_of_a_fused_projection(V):
    """x as channels of a wider row, dx into channels of a wider gradient, whose other channels stay."""
    import torch
    B, L, H, d = 2, 9, 3, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    fused = torch.randn(B, L, 5 * H * d, generator=g, device="cuda")
    f = torch.rand(16, generator=g, device="cuda")
    part = fused[:, :, H * d:2 * H * d]
    kw = dict(grid=(3, 3), l2=True)
    y = V.rope(part, f, (4, 6, 6), H, **kw)
    assert torch.equal(y, V.rope(part.contiguous(), f, (4, 6, 6), H, **kw))
    dfused = torch.full_like(fused, 3.0)
    dx = V.rope_backward(y, f, (4, 6, 6), H, x=part, out=dfused[:, :, H * d:2 * H * d], **kw)
    assert torch.equal(dx, V.rope_backward(y, f, (4, 6, 6), H, x=part.contiguous(), **kw))
    assert (dfused[:, :, :H * d] == 3).all() and (dfused[:, :, 2 * H * d:] == 3).all()
    with pytest.raises(ValueError):
        V.rope(fused[:, ::2, :H * d].expand(B, -1, -1)[:, :, ::2], f, (4, 6, 6), H, grid=(3, 3))
    with pytest.raises(ValueError):  # rows not at one stride over the batch
        V.rope(fused[:, :4, :H * d], f, (4, 6, 6), H, grid=(3, 3))


def test_tensors_past_32_bits(V):
    """The last tokens of more than 2^31 elements, as by themselves."""
    import torch
    H, d, L = 16, 128, (1 << 20) + 70
    x = torch.empty(1, L, H * d, dtype=torch.bfloat16, device="cuda").normal_(0, 1)
    f = torch.rand(64, device="cuda")
    last = x[:, -70:].contiguous()
    kw = dict(l2=True, layout="heads")
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[None, :, None].expand(1, L, 3).contiguous()
    y = V.rope(x, f, (16, 24, 24), H, positions=pos, **kw)
    want = V.rope(last, f, (16, 24, 24), H, positions=pos[:, -70:].contiguous(), **kw)
    assert torch.equal(y[:, -70:], want)
    dx = V.rope_backward(y, f, (16, 24, 24), H, x=x, positions=pos, **kw)
    dlast = V.rope_backward(want, f, (16, 24, 24), H, x=last, positions=pos[:, -70:].contiguous(), **kw)
    assert torch.equal(dx[:, -70:], dlast)


def test_other_stream_and_graph(V):
    import torch
    x = torch.randn(1, 77, 4 * 64, device="cuda").bfloat16()
    f = torch.rand(32, device="cuda")
    kw = dict(grid=(7, 11), l2=True)
    want = V.rope(x, f, (8, 12, 12), 4, **kw)
    back = V.rope_backward(want, f, (8, 12, 12), 4, x=x, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = V.rope(x, f, (8, 12, 12), 4, stream=side, **kw)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = V.rope(x, f, (8, 12, 12), 4, **kw)
        dx = V.rope_backward(y, f, (8, 12, 12), 4, x=x, **kw)
    for turn in range(3):
        y.zero_(), dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, back), turn


def test_argument_errors(V):
    import torch
    x = torch.randn(2, 6, 2 * 32, device="cuda")
    f = torch.rand(16, device="cuda")
    p = torch.zeros(2, 6, 3, dtype=torch.int32, device="cuda")
    ok = dict(positions=p)
    V.rope(x, f, (4, 6, 6), 2, **ok)
    for args, kw in [((x, f[:8], (4, 6, 6), 2), ok), ((x, f, (4, 6, 6), 3), ok), ((x, f, (4, 6, 6), 2), {}),
                     ((x, f, (4, 6, 6), 2), dict(positions=p.long())), ((x, f, (4, 6, 6), 2), dict(positions=p, grid=(2, 3))),
                     ((x, f, (4, 6, 6), 2), dict(ok, layout="x")), ((x.half(), f, (4, 6, 6), 2), ok),
                     ((x, f.double(), (4, 6, 6), 2), ok), ((x, f, (-4, 14, 6), 2), ok),
                     ((x, f[:12].contiguous(), (4, 4, 4), 2), ok)]:
        with pytest.raises(ValueError):
            V.rope(*args, **kw)
    with pytest.raises(ValueError):
        V.rope_backward(x.view(4, 6, 32), f, (4, 6, 6), 2, l2=True, **ok)
