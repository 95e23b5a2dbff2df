"""A captured serving step: the recurrence's and the cross attention's tokens, one graph
replayed token by token, with the program's own eager work between the replays."""
import numpy as np
import pytest

import oracle.cross_oracle as X
import oracle.recur_oracle as R
from test_gpu_cross import HALF, V, _hold  # noqa: F401  (V: the fixture)
from vda_testutil import from_device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [90, 3000], ids=["one_launch", "joined"])
def test_captured_step(V, S):
    import torch
    n, m, H, d, tokens = 4, 6, 4, 64, 5
    C = H * d
    rng = np.random.default_rng(S)
    xs, gs = (torch.from_numpy(rng.standard_normal((tokens, n, 1, C))).bfloat16() for _ in range(2))
    k, v = (torch.from_numpy(rng.standard_normal((m, S, H, d))).bfloat16() for _ in range(2))
    lens = [S, S // 2, 1, 0, S - 1, 40]
    first = torch.from_numpy(rng.standard_normal((m, C))).float()
    # Slots of each token's sequences: they move, and some rows are padding.
    slots = [[0, 1, 2, 3], [0, 1, 2, 3], [5, -1, 2, 3], [5, 4, 2, m], [1, 4, 0, 3]]
    x, g = (torch.zeros(n, 1, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = torch.zeros(n, dtype=torch.int32, device="cuda")
    state = first.cuda()
    kc, vc, kl = k.cuda(), v.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    h = torch.full((n, 1, C), 9.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((n, 1, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
    need = V.cross_step_workspace(h.view(n, 1, H, d), kc, vc)
    assert (need > 0) == (S == 3000)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def step():
        V.recur_step(x, g, state, gate="logit", slots=at, out=h)
        V.cross_step(h.view(n, 1, H, d), kc, vc, k_lens=kl, slots=at, out=out, work=work)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    at.fill_(-1)
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    half, S64 = HALF["bf16"], first.double().numpy()
    for t in range(tokens):
        x.copy_(xs[t]), g.copy_(gs[t]), at.copy_(torch.tensor(slots[t], dtype=torch.int32))
        h.fill_(9.0), out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got_h, got, after = from_device(h), from_device(out), from_device(state)
        for i, slot in enumerate(slots[t]):
            if slot < 0 or slot >= m:
                assert (got_h[i] == 9.0).all() and (got[i] == 9.0).all()
                continue
            a = (xs[t, i].double().numpy(), gs[t, i].double().numpy(), "logit", S64[slot])
            (want, last), (b, bl) = R.recur_sequence(*a), R.recur_bounds(*a, half)
            _hold(got_h[i], want, b, (t, i, "h"))
            _hold(after[slot], last, bl, (t, i, "state"))
            q = got_h[i].reshape(1, H, d)  # what the second call reads
            a = (q, k[slot].double().numpy(), v[slot].double().numpy(), np.arange(S) < lens[slot], d ** -0.5)
            _hold(got[i], X.cross_sequence(*a)[0], X.cross_bounds(*a, half)[0], (t, i, "out"))
        untouched = sorted(set(range(m)) - set(slots[t]))
        assert (after[untouched] == S64[untouched]).all()
        S64 = after
        # Eager work of the program on the same tensors' stream, between replays.
        V.cross_step(h.view(n, 1, H, d), kc, vc, k_lens=kl, slots=at)
        torch.cuda.synchronize()
