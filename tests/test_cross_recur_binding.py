"""Checks of the cross attention's and the recurrence's Python binding: sizes that the C
entry points do not see as they are, because their arguments are 32-bit, are refused
before the call.  (Tensors without memory; the calls are recorded in place of made.)"""
import pytest
import torch

vda = pytest.importorskip("paper_2609_20744_amd.vda", reason="libvda.so not built")

PAST = 1 << 32


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(vda, "_storage", lambda t, name: (t.dtype, t.device))
    monkeypatch.setattr(vda, "_stream_ptr", lambda dev, stream=None: 0)
    monkeypatch.setattr(vda, "_call", lambda fn, dev, *args: made.append(args) or 0)
    return made


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def _step(n=3, t=2, C=8, m=5):
    return vda.recur_step(_meta(n, t, C), _meta(n, t, C), _meta(m, C, dtype=torch.float32), gate="logit",
                          slots=_meta(n, dtype=torch.int32))


@pytest.mark.parametrize("kw", [dict(m=PAST + 5), dict(m=(1 << 31) + 5), dict(n=PAST + 3), dict(t=PAST + 2), dict(C=PAST + 8)], ids=str)
def test_recur_step(calls, kw):
    """Not taken modulo 2^32, in which each of these is a sound call (of a pool of five slots, the others padding)."""
    _step()
    assert calls[-1][2:5] == (3, 2, 8)
    del calls[:]
    with pytest.raises(ValueError):
        _step(**kw)
    assert not calls


@pytest.mark.parametrize("kw", [dict(d=PAST + 64), dict(Hq=PAST + 4), dict(Hq=PAST + 4, Hk=PAST + 2), dict(L=PAST + 4), dict(S=PAST + 6),
                                dict(n=PAST + 2)], ids=str)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_cross(calls, layout, kw):
    def sides(n=2, L=4, S=6, Hq=4, Hk=2, d=64):
        if layout == "heads":
            return _meta(n, Hq, L, d), _meta(n, Hk, S, d), _meta(n, Hk, S, d)
        return _meta(n, L, Hq, d), _meta(n, S, Hk, d), _meta(n, S, Hk, d)

    vda.cross_forward(*sides(), layout=layout)
    assert calls
    del calls[:]
    with pytest.raises(ValueError):
        vda.cross_forward(*sides(**kw), layout=layout)
    with pytest.raises(ValueError):
        vda.cross_workspace(*sides(**kw), layout=layout)
    assert not calls


@pytest.mark.parametrize("kw", [dict(d=PAST + 64), dict(Hq=PAST + 4), dict(t=PAST + 2), dict(S=PAST + 6), dict(n=PAST + 2),
                                dict(m=PAST + 5)], ids=str)
def test_cross_step(calls, kw):
    def sides(n=3, t=2, m=5, S=6, Hq=4, Hk=2, d=64):
        return _meta(n, t, Hq, d), _meta(m, S, Hk, d), _meta(m, S, Hk, d)

    vda.cross_step(*sides())
    del calls[:]
    with pytest.raises(ValueError):
        vda.cross_step(*sides(**kw))
    assert not calls


@pytest.mark.parametrize("kw", [dict(n=PAST + 2), dict(L=PAST + 4), dict(C=PAST + 8)], ids=str)
def test_recur(calls, kw):
    def args(n=2, L=4, C=8):
        return _meta(n, L, C), _meta(n, L, C)

    vda.recur_forward(*args(), gate="logit")
    del calls[:]
    with pytest.raises(ValueError):
        vda.recur_forward(*args(**kw), gate="logit")
    with pytest.raises(ValueError):
        vda.recur_workspace(*args(**kw), gate="logit")
    assert not calls


def test_sequences_of_a_packed_batch(calls):
    cu = _meta(PAST + 3, dtype=torch.int32)  # two sequences, modulo 2^32
    with pytest.raises(ValueError):
        vda.cross_forward(_meta(4, 2, 64), _meta(6, 2, 64), _meta(6, 2, 64), cu_q=cu, cu_k=cu, layout="tokens")
    with pytest.raises(ValueError):
        vda.recur_forward(_meta(4, 8), _meta(4, 8), gate="logit", cu_seqlens=cu)
    assert not calls
