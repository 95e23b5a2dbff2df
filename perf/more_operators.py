"""Calls of cross attention to an encoder's states and of the gated linear recurrence, and the ranges they stand for.

A case names one operator (``op``) with its sizes, storage type and options:

* ``cross``: softmax attention of a sequence's queries to the states of an encoder, of another length
  (``vda.cross_forward``); ``cross_bwd``: its gradients (``vda.cross_backward``); ``cross_step``: a few tokens of each
  sequence against a pool of cached states (``vda.cross_step``);
* ``recur``: the channel-wise gated recurrence over whole sequences (``vda.recur_forward``); ``recur_bwd``: its gradients
  (``vda.recur_backward``); ``recur_step``: a few tokens of each sequence of a state pool (``vda.recur_step``).

Per query head h, with key head h / (H_q / H_k) and the keys j that the sequence's length and mask leave,

    s_j = scale q . k_j,   lse = log sum_j exp(s_j),   out = sum_j exp(s_j - lse) v_j      (no key left: 0, lse = -inf).

Per channel, h_t = a_t h_{t-1} + u_t, out_t = h_t, with (``gate``) a = exp(g), u = x (``log``); a = sigmoid(g),
u = (1 - a) x (``logit``); a = sigmoid(g), u = sqrt(1 - a^2) x (``norm``); ``reverse`` takes the tokens from the last.
"""
import math

import torch

own = False


def _case(name, op, **kw):
    base = {"name": name, "op": op, "dtype": "bf16"}
    if op == "cross_step":
        base.update(n=1, t=1, slots=1, S=1, Hq=1, Hk=1, d=128, kv_layout="tokens", uneven=False)
    elif op in ("cross", "cross_bwd"):
        base.update(n=1, T=1, S=1, Hq=1, Hk=1, d=128, layout="tokens", kv_layout="tokens", ragged=False, uneven=False,
                    mask=False)
    elif op == "recur_step":
        base.update(n=1, t=1, slots=1, C=8, gate="log")
    else:
        base.update(n=1, T=1, C=8, gate="log", ragged=False, state=False, reverse=False)
    base.update(kw)
    return base


def listed():
    return [
        # One stream, one token, one prompt of 512 states: the smallest serving call, where latency decides.
        _case("cross_one", "cross_step", n=1, slots=4, S=512, Hq=16, Hk=16),
        # A full batch of streams, a token each, four query heads to a key head; prompts of uneven length in a pool of
        # 2048 states a slot, some of them shared, some rows padding.
        _case("cross_batch", "cross_step", n=96, slots=112, S=2048, Hq=32, Hk=8, uneven=True),
        # A whole 480p clip (21 frames of 30 x 52) of 24 heads reads a prompt of 512 states: the largest product.
        _case("cross_clip", "cross", T=32760, S=512, Hq=24, Hk=24, layout="heads"),
        # Requests of uneven length packed into one call, each with its own states, some of those masked out.
        _case("cross_packed", "cross", n=24, T=16411, S=9601, Hq=16, Hk=8, ragged=True, mask=True),
        # 64 learned queries of each of two clips read ten 768p frames (48 x 84): few rows, long states.
        _case("cross_few", "cross", n=2, T=128, S=80640, Hq=16, Hk=16, d=64),
        # A small training step in fp32: what a user checks a bf16 run against. Prompts padded to one length.
        _case("cross_bwd_f32", "cross_bwd", dtype="f32", n=2, T=666, S=154, Hq=4, Hk=4, d=64, uneven=True),
        # A training step over packed clips, two query heads to a key head, masked states.
        _case("cross_bwd_packed", "cross_bwd", n=9, T=16401, S=4607, Hq=16, Hk=8, ragged=True, mask=True),
        # A token of each of 192 streams, states in a pool.
        _case("recur_batch", "recur_step", n=192, slots=224, C=2048, gate="logit"),
        # Ten 768p frames of one clip, the 896 channels of a 7-head shard: one long sequence, few channels.
        _case("recur_long", "recur", T=40320, C=896),
        # Requests of uneven length packed into one call, read from their ends, states in and out.
        _case("recur_packed", "recur", n=24, T=16411, C=2048, gate="norm", ragged=True, state=True, reverse=True),
        # A small training step in fp32.
        _case("recur_bwd_f32", "recur_bwd", dtype="f32", n=2, T=666, C=256, gate="logit"),
        # A training step over packed clips with the state's gradient.
        _case("recur_bwd_packed", "recur_bwd", n=9, T=16401, C=2048, gate="logit", ragged=True, state=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call: any operator, sizes over the whole range (odd ones among them), any options."""
    op = rng.choice(["cross"] * 4 + ["cross_bwd"] * 3 + ["cross_step"] * 3 + ["recur"] * 3 + ["recur_bwd"] * 3 + ["recur_step"])
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op.startswith("cross"):
        Hk = rng.randint(1, 16)
        Hq = Hk * rng.choice([1, 1, 2, 4])
        d = rng.choice([128, 128, 64, 64, 32])
        kv = rng.choice(["heads", "tokens"])
        if op == "cross_step":
            most = 96 * 2048 * 8 * 128 // (Hk * d) // (1 if dt == "bf16" else 2)  # states read
            n = _log_int(rng, 1, 96)
            c = _case("", op, dtype=dt, n=n, t=rng.choice([1, 1, 1, 2, 5]), slots=n + rng.randint(0, 16),
                      S=_log_int(rng, 1, max(1, min(20000, most // n))), Hq=Hq, Hk=Hk, d=d, kv_layout=kv,
                      uneven=rng.random() < 0.6)
        else:
            most = 32760 * 512 * 24 * 128 // (Hq * d) // (3 if op == "cross_bwd" else 1)  # pairs of query and key
            if dt == "f32":
                most //= 8
            T = _log_int(rng, 1, 32760)
            S = _log_int(rng, 1, max(1, min(80640, most // T)))
            n = min(T, S, rng.choice([1, 1, 2, 5, 24]))
            ragged = n > 1 and rng.random() < 0.6
            c = _case("", op, dtype=dt, n=n, T=T if ragged else T // n * n, S=S if ragged else S // n * n, Hq=Hq, Hk=Hk, d=d,
                      layout=rng.choice(["heads", "tokens"]), kv_layout=kv, ragged=ragged,
                      uneven=not ragged and rng.random() < 0.5, mask=rng.random() < 0.4)
    else:
        C = 8 * _log_int(rng, 1, 512)
        gate = rng.choice(["log", "logit", "norm"])
        if op == "recur_step":
            n = _log_int(rng, 1, 256)
            c = _case("", op, dtype=dt, n=n, t=rng.choice([1, 1, 2, 5]), slots=n + rng.randint(0, 32), C=C, gate=gate)
        else:
            most = 40320 * 896 // (1 if dt == "bf16" else 2)
            T = _log_int(rng, 1, min(40320 if op == "recur" else 16401, most // C))
            n = min(T, rng.choice([1, 1, 2, 5, 24]))
            ragged = n > 1 and rng.random() < 0.6
            c = _case("", op, dtype=dt, n=n, T=T if ragged else T // n * n, C=C, gate=gate, ragged=ragged,
                      state=rng.random() < 0.5, reverse=rng.random() < 0.5)
    del c["name"]
    return c


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------

KEEP = 0.9  # share of the states that a mask leaves
HALF = 0.55  # mean share of a padded length that its sequence fills


def _cuts(total, n, gen):
    """Offsets of n uneven sequences of `total` tokens, short and empty ones among them."""
    w = torch.rand(n, generator=gen, device="cuda").double() ** 2 + 0.01
    if n >= 6:
        w[n // 3] = 0.0
    cu = (w.cumsum(0) / w.sum() * total).round().to(torch.int32)
    cu[-1] = total
    return torch.cat([cu.new_zeros(1), cu])


def _filled(n, most, gen):
    """Lengths of n padded sequences, the last of three or more empty."""
    f = 0.1 + 2 * (HALF - 0.1) * torch.rand(n, generator=gen, device="cuda")
    lens = (f * most).round().clamp(1, most).to(torch.int32)
    if n >= 3:
        lens[-1] = 0
    return lens


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, op, n = _dtype(case), case["op"], case["n"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": case}
    if op.startswith("recur"):
        C = case["C"]
        lead = (n, case["t"]) if op == "recur_step" else (case["T"],) if case["ragged"] else (n, case["T"] // n)
        s["x"] = randn(*lead, C).to(dt)
        # Channels of short and of long memory, as their biases settle; gates vary about them.
        bias = 6.0 * rand(C) - 1.0
        z = bias + randn(*lead, C)
        if case["gate"] == "log":
            z = -torch.nn.functional.softplus(-z)
            s["g"] = torch.where(rand(*lead, 1) < 0.002, -math.inf, z)  # some tokens reset the state
        else:
            s["g"] = z.to(dt)
        if op == "recur_step":
            s["state"] = randn(case["slots"], C)
            slots = torch.randperm(case["slots"], generator=g, device="cuda")[:n].to(torch.int32)
            slots[1:][rand(n - 1) < 0.06] = -1
            s["slots"], s["out"] = slots, torch.zeros_like(s["x"])
            return s
        s["cu"] = _cuts(case["T"], n, g) if case["ragged"] else None
        s["state"] = randn(n, C) if case["state"] else None
        if op == "recur_bwd":
            s["dout"] = randn(*lead, C).to(dt)
            s["dstate"] = randn(n, C) if case["state"] else None
        return s

    Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
    s["scale"] = d ** -0.5
    if op == "cross_step":
        m, S = case["slots"], case["S"]
        s["q"] = 1.5 * randn(n, case["t"], Hq, d)
        shape = (m, Hk, S, d) if case["kv_layout"] == "heads" else (m, S, Hk, d)
        s["k"], s["v"] = randn(*shape).to(dt), randn(*shape).to(dt)
        s["q"] = s["q"].to(dt)
        s["k_lens"] = _filled(m, S, g) if case["uneven"] else None
        # Streams of one prompt share its slot; a few rows are padding.
        slots = torch.randint(0, m, (n,), generator=g, device="cuda", dtype=torch.int32)
        slots[1:][rand(n - 1) < 0.06] = -1
        s["slots"], s["out"] = slots, torch.zeros_like(s["q"])
        return s

    def shape(layout, total, H):
        if case["ragged"]:
            return (H, total, d) if layout == "heads" else (total, H, d)
        return (n, H, total // n, d) if layout == "heads" else (n, total // n, H, d)

    T, S = case["T"], case["S"]
    s["q"] = (1.5 * randn(*shape(case["layout"], T, Hq))).to(dt)
    s["k"], s["v"] = (randn(*shape(case["kv_layout"], S, Hk)).to(dt) for _ in range(2))
    s["cu_q"], s["cu_k"] = (_cuts(T, n, g), _cuts(S, n, g)) if case["ragged"] else (None, None)
    s["k_lens"] = _filled(n, S // n, g) if case["uneven"] else None
    s["k_mask"] = None
    if case["mask"]:
        s["k_mask"] = rand(*((S,) if case["ragged"] else (n, S // n))) < KEEP
        # What stands in a masked place may be anything.
        hidden = ~s["k_mask"]
        hidden = hidden[..., None, None] if case["kv_layout"] == "tokens" else hidden[..., None, :, None]
        s["k"].masked_fill_(hidden, math.inf)
        s["v"].masked_fill_(hidden, math.nan)
    if op == "cross_bwd":
        s["dout"] = randn(*s["q"].shape).to(dt)
        s.update(_plain_cross(s))  # a training program has the forward pass's output and lse
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------------------------------------------------

def _lengths(cu, n, total):
    """First token and length of each sequence."""
    if cu is None:
        return torch.arange(n, device="cuda") * (total // n), torch.full((n,), total // n, device="cuda")
    return cu[:-1].long(), (cu[1:] - cu[:-1]).long()


def _gather(x, layout, cu, n, total, most):
    """[n, H, most, d] fp32 of a packed or batched tensor, and which places are real [n, most]."""
    at, lens = _lengths(cu, n, total)
    i = torch.arange(most, device="cuda")
    real = i < lens[:, None]
    if cu is None:
        return (x if layout == "heads" else x.transpose(1, 2)).float(), real
    x = x.transpose(0, 1) if layout == "heads" else x
    return x[(at[:, None] + i).clamp(max=total - 1)].float().transpose(1, 2), real


def _scatter(x, like, layout, cu, real):
    """The inverse of _gather, in the type of `like`."""
    if cu is None:
        return (x if layout == "heads" else x.transpose(1, 2)).to(like.dtype).contiguous()
    x = x.transpose(1, 2)[real]
    return (x.transpose(0, 1) if layout == "heads" else x).to(like.dtype).contiguous()


def _most(cu, n, total):
    return total // n if cu is None else int((cu[1:] - cu[:-1]).max())


def _softmax(sc):
    """exp(s - lse) and lse along the last axis; a row of -inf gives zeros and -inf."""
    m = sc.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = (sc - m).exp()
    l = p.sum(-1, keepdim=True)
    return p / l.clamp(min=1e-30), (m + l.log())[..., 0]


def _cross_parts(s):
    """q and the sequences' keys and values of every query head, scores with -inf where a key is not seen."""
    case, n = s["case"], s["case"]["n"]
    lq, lk = _most(s["cu_q"], n, case["T"]), _most(s["cu_k"], n, case["S"])
    q, real = _gather(s["q"], case["layout"], s["cu_q"], n, case["T"], lq)
    k, seen = _gather(s["k"], case["kv_layout"], s["cu_k"], n, case["S"], lk)
    v, _ = _gather(s["v"], case["kv_layout"], s["cu_k"], n, case["S"], lk)
    keys = seen
    if s["k_lens"] is not None:
        seen = seen & (torch.arange(lk, device="cuda") < s["k_lens"][:, None])
    if s["k_mask"] is not None:
        m = s["k_mask"]
        if s["cu_k"] is not None:
            m = m[(s["cu_k"][:-1].long()[:, None] + torch.arange(lk, device="cuda")).clamp(max=case["S"] - 1)]
        seen = seen & m
    group = case["Hq"] // case["Hk"]
    k, v = (torch.where(seen[:, None, :, None], x, 0.0).repeat_interleave(group, 1) for x in (k, v))
    sc = (s["scale"] * (q @ k.transpose(-1, -2))).masked_fill(~seen[:, None, None, :], -math.inf)
    return q, k, v, sc, real, keys


def _plain_cross(s):
    case = s["case"]
    q, k, v, sc, real, _ = _cross_parts(s)
    p, lse = _softmax(sc)
    lse = lse if s["cu_q"] is None else lse.transpose(1, 2)[real].transpose(0, 1).contiguous()
    return {"out": _scatter(p @ v, s["q"], case["layout"], s["cu_q"], real), "lse": lse}


def _plain_cross_bwd(s):
    case = s["case"]
    q, k, v, sc, real, keys = _cross_parts(s)
    p, _ = _softmax(sc)
    do, _ = _gather(s["dout"], case["layout"], s["cu_q"], case["n"], case["T"], q.shape[2])
    do, q = (torch.where(real[:, None, :, None], x, 0.0) for x in (do, q))
    dp = do @ v.transpose(-1, -2)
    ds = s["scale"] * p * (dp - (p * dp).sum(-1, keepdim=True))
    group = case["Hq"] // case["Hk"]
    dk, dv = (x.unflatten(1, (-1, group)).sum(2) for x in (ds.transpose(-1, -2) @ q, p.transpose(-1, -2) @ do))
    return {"dq": _scatter(ds @ k, s["q"], case["layout"], s["cu_q"], real),
            "dk": _scatter(dk, s["k"], case["kv_layout"], s["cu_k"], keys),
            "dv": _scatter(dv, s["v"], case["kv_layout"], s["cu_k"], keys)}


def _plain_cross_step(s):
    case = s["case"]
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    at, group = s["slots"][rows].long(), case["Hq"] // case["Hk"]
    k, v = (x if case["kv_layout"] == "heads" else x.transpose(1, 2) for x in (s["k"], s["v"]))
    k, v = k[at].float(), v[at].float()
    q = s["q"][rows].float().transpose(1, 2).reshape(len(at), case["Hk"], -1, case["d"])  # a key head's queries
    sc = s["scale"] * (q @ k.transpose(-1, -2))
    if s["k_lens"] is not None:
        sc = sc.masked_fill(torch.arange(case["S"], device="cuda") >= s["k_lens"][at][:, None, None, None], -math.inf)
    p, _ = _softmax(sc)
    o = (p @ v).reshape(len(at), case["Hk"] * group, case["t"], case["d"]).transpose(1, 2)
    s["out"][rows] = o.to(s["out"].dtype)
    return {"out": s["out"]}


def _gates(x, g, gate):
    """a and u in fp32."""
    x, g = x.float(), g.float()
    if gate == "log":
        return g.exp(), x
    a, b = g.sigmoid(), (-g).sigmoid()
    return a, (b if gate == "logit" else (b * (1 + a)).sqrt()) * x


def _scan(a, u, first):
    """h_t = a_t h_{t-1} + u_t along axis 1 of [n, L, C], from `first` [n, C]; steps of doubled length."""
    u = torch.cat([u[:, :1] + a[:, :1] * first[:, None], u[:, 1:]], 1) if u.shape[1] else u
    step = 1
    while step < u.shape[1]:
        u = torch.cat([u[:, :step], u[:, step:] + a[:, step:] * u[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return u


def _rows(s, x):
    """[n, most, C] of a packed or batched tensor, the tokens in the order of the recurrence, and which are real."""
    case, n = s["case"], s["case"]["n"]
    at, lens = _lengths(s["cu"], n, case["T"])
    i = torch.arange(_most(s["cu"], n, case["T"]), device="cuda")
    real = i < lens[:, None]
    i = (lens[:, None] - 1 - i) if case["reverse"] else i.expand(n, -1)
    i = (at[:, None] + i).clamp(0, max(case["T"] - 1, 0))
    return x.reshape(-1, case["C"])[i], real, i


def _back(s, x, real, i, like):
    out = torch.empty_like(like)
    out.view(-1, s["case"]["C"])[i[real]] = x[real].to(like.dtype)
    return out


def _recur_parts(s):
    case = s["case"]
    x, real, i = _rows(s, s["x"])
    g, _, _ = _rows(s, s["g"])
    a, u = _gates(x, g, case["gate"])
    a, u = torch.where(real[..., None], a, 1.0), torch.where(real[..., None], u, 0.0)  # a place behind the end keeps the state
    first = s["state"] if s["state"] is not None else torch.zeros(case["n"], case["C"], device="cuda")
    return x.float(), g.float(), real, i, a, first, _scan(a, u, first)


def _plain_recur(s):
    _, _, real, i, _, first, h = _recur_parts(s)
    return {"out": _back(s, h, real, i, s["x"]), "state": h[:, -1] if h.shape[1] else first}


def _plain_recur_bwd(s):
    case = s["case"]
    x, g, real, i, a, first, h = _recur_parts(s)
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    do = torch.where(real[..., None], _rows(s, s["dout"])[0].float(), 0.0)
    last = s["dstate"] if s["dstate"] is not None else torch.zeros_like(first)
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    dh = _scan(after.flip(1), do.flip(1), last).flip(1)
    if case["gate"] == "log":
        dx, dg = dh, dh * a * before
    else:
        b = (-g).sigmoid()
        if case["gate"] == "logit":
            dx, dg = dh * b, dh * a * b * (before - x)
        else:
            dx, dg = dh * (b * (1 + a)).sqrt(), dh * (a * b * before - a * a * (b / (1 + a)).sqrt() * x)
    return {"dx": _back(s, dx, real, i, s["x"]), "dg": _back(s, dg, real, i, s["g"]),
            "dstate": a[:, 0] * dh[:, 0] if s["state"] is not None else None}


def _plain_recur_step(s):
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    at = s["slots"][rows].long()
    a, u = _gates(s["x"][rows], s["g"][rows], s["case"]["gate"])
    h = _scan(a, u, s["state"][at])
    s["state"][at] = h[:, -1]
    s["out"][rows] = h.to(s["out"].dtype)
    return {"out": s["out"], "state": s["state"]}


def run(s):
    case = s["case"]
    if not own:
        return {"cross": _plain_cross, "cross_bwd": _plain_cross_bwd, "cross_step": _plain_cross_step,
                "recur": _plain_recur, "recur_bwd": _plain_recur_bwd, "recur_step": _plain_recur_step}[case["op"]](s)
    from paper_2609_20744_amd import vda
    if case["op"] == "recur_step":
        out = vda.recur_step(s["x"], s["g"], s["state"], gate=case["gate"], slots=s["slots"], out=s["out"])
        return {"out": out, "state": s["state"]}
    if case["op"] == "cross_step":
        return {"out": vda.cross_step(s["q"], s["k"], s["v"], k_lens=s["k_lens"], slots=s["slots"], kv_layout=case["kv_layout"],
                                      scale=s["scale"], out=s["out"])}
    if case["op"].startswith("recur"):
        opts = dict(gate=case["gate"], cu_seqlens=s["cu"], reverse=case["reverse"], state=s["state"])
        if case["op"] == "recur":
            out, state = vda.recur_forward(s["x"], s["g"], return_state=True, **opts)
            return {"out": out, "state": state}
        return dict(zip(("dx", "dg", "dstate"), vda.recur_backward(s["dout"], s["x"], s["g"], dstate=s["dstate"], **opts)))
    opts = dict(cu_q=s["cu_q"], cu_k=s["cu_k"], k_lens=s["k_lens"], k_mask=s["k_mask"], layout=case["layout"],
                kv_layout=case["kv_layout"], scale=s["scale"])
    if case["op"] == "cross":
        out, lse = vda.cross_forward(s["q"], s["k"], s["v"], return_lse=True, **opts)
        return {"out": out, "lse": lse}
    return dict(zip(("dq", "dk", "dv"), vda.cross_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], **opts)))


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    es, n, op = 4 if case["dtype"] == "f32" else 2, case["n"], case["op"]
    if op.startswith("recur"):
        C, ge = case["C"], 4 if case["gate"] == "log" else es
        if op == "recur_step":
            rows = n * case["t"] * C
            return {"bytes": rows * (2 * es + ge) + 8 * n * C, "flops": 8 * rows}
        x, state = case["T"] * C, 4 * n * C
        if op == "recur":
            return {"bytes": x * (2 * es + ge) + state * (2 if case["state"] else 1), "flops": 8 * x}
        return {"bytes": x * (3 * es + 2 * ge) + state * (3 if case["state"] else 0), "flops": 20 * x}
    Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
    if op == "cross_step":
        seen, m = case["S"] * (HALF if case["uneven"] else 1.0), case["slots"]
        read = m * (1 - (1 - 1 / m) ** n)  # slots that some stream has
        return {"bytes": 2 * n * case["t"] * Hq * d * es + 2 * read * seen * Hk * d * es,
                "flops": 4 * n * case["t"] * seen * Hq * d}
    T, S = case["T"], case["S"]
    seen = (HALF if case["uneven"] else 1.0) * (KEEP if case["mask"] else 1.0)
    pairs = T * S / n * seen * Hq
    q, kv, lse = T * Hq * d * es, 2 * S * Hk * d * es, 4 * T * Hq
    if op == "cross":
        return {"bytes": 2 * q + kv * seen + lse, "flops": 4 * pairs * d}
    return {"bytes": 4 * q + kv * seen + kv + lse, "flops": 10 * pairs * d}


def _sequences(s):
    """Slices of each sequence's queries and keys, and which of its keys are seen."""
    case, n = s["case"], s["case"]["n"]
    cq = s["cu_q"].tolist() if case["ragged"] else [case["T"] // n * i for i in range(n + 1)]
    ck = s["cu_k"].tolist() if case["ragged"] else [case["S"] // n * i for i in range(n + 1)]
    mask = s["k_mask"].flatten() if s["k_mask"] is not None else torch.ones(case["S"], dtype=torch.bool, device="cuda")
    for i in range(n):
        seen = mask[ck[i]:ck[i + 1]].clone()
        if s["k_lens"] is not None:
            seen[int(s["k_lens"][i]):] = False
        yield slice(cq[i], cq[i + 1]), slice(ck[i], ck[i + 1]), seen


def _flat(x, layout, ragged):
    """[tokens, H, d] in 64 bits."""
    if layout == "tokens":
        return x.double().flatten(0, -3)
    return x.double().transpose(0, 1) if ragged else x.double().transpose(1, 2).flatten(0, 1)


def _unflat(x, like, layout, ragged):
    if layout == "tokens":
        return x.reshape(like.shape)
    return x.transpose(0, 1).contiguous() if ragged else x.unflatten(0, (like.shape[0], -1)).transpose(1, 2).contiguous()


def _exact_cross(s):
    """One sequence and one key head at a time, over the keys that it sees."""
    case, bwd = s["case"], s["case"]["op"] == "cross_bwd"
    group = case["Hq"] // case["Hk"]
    q = _flat(s["q"], case["layout"], case["ragged"])
    k, v = (_flat(s[x], case["kv_layout"], case["ragged"]) for x in ("k", "v"))
    do = _flat(s["dout"], case["layout"], case["ragged"]) if bwd else None
    out, lse = torch.zeros_like(q), q.new_full(q.shape[:2], -math.inf)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for rows, cols, seen in _sequences(s):
        if rows.stop == rows.start or not bool(seen.any()):
            continue
        at = cols.start + seen.nonzero()[:, 0]
        for h in range(case["Hk"]):
            heads = slice(h * group, (h + 1) * group)
            qi, ki, vi = q[rows, heads].flatten(0, 1), k[at, h], v[at, h]
            sc = s["scale"] * (qi @ ki.T)
            z = torch.logsumexp(sc, -1)
            p = (sc - z[:, None]).exp()
            oi = p @ vi
            out[rows, heads], lse[rows, heads] = oi.unflatten(0, (-1, group)), z.unflatten(0, (-1, group))
            if bwd:
                di = do[rows, heads].flatten(0, 1)
                ds = s["scale"] * p * (di @ vi.T - (di * oi).sum(-1, keepdim=True))
                dq[rows, heads] = (ds @ ki).unflatten(0, (-1, group))
                dk[at, h], dv[at, h] = ds.T @ qi, p.T @ di
    if bwd:
        return {"dq": _unflat(dq, s["q"], case["layout"], case["ragged"]),
                "dk": _unflat(dk, s["k"], case["kv_layout"], case["ragged"]),
                "dv": _unflat(dv, s["v"], case["kv_layout"], case["ragged"])}
    lse = lse.T.contiguous() if case["ragged"] else lse.unflatten(0, (case["n"], -1)).transpose(1, 2).contiguous()
    return {"out": _unflat(out, s["q"], case["layout"], case["ragged"]), "lse": lse}


def _exact_cross_step(s):
    """One row, then one key head at a time."""
    case = s["case"]
    group, out = case["Hq"] // case["Hk"], s["out"].double()
    for i, slot in enumerate(s["slots"].tolist()):
        m = case["S"] if s["k_lens"] is None or slot < 0 else int(s["k_lens"][slot])
        if slot < 0:
            continue
        k, v = (x[slot].double() if case["kv_layout"] == "heads" else x[slot].double().transpose(0, 1) for x in (s["k"], s["v"]))
        for h in range(case["Hk"]):
            heads = slice(h * group, (h + 1) * group)
            p = torch.softmax(s["scale"] * (s["q"][i, :, heads].double() @ k[h, :m].T), -1)
            out[i, :, heads] = p @ v[h, :m]
    return {"out": out}


def _token_gates(x, g, gate):
    """a, u, their derivatives by g, and u's by x, in 64 bits."""
    x, g = x.double(), g.double()
    if gate == "log":
        a = g.exp()
        return a, x, a, torch.zeros_like(x), torch.ones_like(x)
    a, b = torch.sigmoid(g), torch.sigmoid(-g)
    if gate == "logit":
        return a, b * x, a * b, -a * b * x, b
    w = (b * (1 + a)).sqrt()
    return a, w * x, a * b, -a * a * (b / (1 + a)).sqrt() * x, w


def _exact_recur(s):
    """Token by token, the sequences side by side; back over the tokens for the gradients."""
    case, n, C = s["case"], s["case"]["n"], s["case"]["C"]
    cu = s["cu"].tolist() if case["ragged"] else [case["T"] // n * i for i in range(n + 1)]
    order = [list(range(a, b))[::-1] if case["reverse"] else list(range(a, b)) for a, b in zip(cu[:-1], cu[1:])]
    most = max(len(o) for o in order)
    live = [torch.tensor([i for i in range(n) if t < len(order[i])], device="cuda") for t in range(most)]
    where = [torch.tensor([o[t] for o in order if t < len(o)], device="cuda") for t in range(most)]
    a, u, da, du, w = _token_gates(s["x"].reshape(-1, C), s["g"].reshape(-1, C), case["gate"])
    h = s["state"].double().clone() if s["state"] is not None else torch.zeros(n, C, device="cuda", dtype=torch.double)
    out, before = torch.zeros_like(a), torch.zeros_like(a)
    for rows, at in zip(live, where):
        before[at] = h[rows]
        out[at] = torch.addcmul(u[at], a[at], h[rows])
        h[rows] = out[at]
    if case["op"] == "recur":
        return {"out": out.reshape(s["x"].shape), "state": h}
    D = s["dstate"].double().clone() if s["dstate"] is not None else torch.zeros_like(h)
    e = s["dout"].double().reshape(-1, C).clone()
    for rows, at in zip(reversed(live), reversed(where)):
        e[at] += D[rows]
        D[rows] = a[at] * e[at]
    return {"dx": (w * e).reshape(s["x"].shape), "dg": (e * (da * before + du)).reshape(s["g"].shape),
            "dstate": D if s["state"] is not None else None}


def _exact_recur_step(s):
    out, state = s["out"].double(), s["state"].double()
    for i, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            for t in range(s["case"]["t"]):
                a, u, _, _, _ = _token_gates(s["x"][i, t], s["g"][i, t], s["case"]["gate"])
                state[slot] = a * state[slot] + u
                out[i, t] = state[slot]
    return {"out": out, "state": state}


def exact(case, seed):
    s = prepare(case, seed)
    return {"cross": _exact_cross, "cross_bwd": _exact_cross, "cross_step": _exact_cross_step, "recur": _exact_recur,
            "recur_bwd": _exact_recur, "recur_step": _exact_recur_step}[case["op"]](s)
