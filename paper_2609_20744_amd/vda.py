"""Thin Python binding of libvda.so (the C ABI in include/vda.h).

Argument marshalling only: every step of the operator runs in the HIP
kernels of libvda.so.  PyTorch supplies device memory and the stream.
Importing this module raises ImportError if the library is not built.

Tensor layout (batch and heads folded into one leading axis, or kept as any
number of leading axes, which are flattened):
    q, k  [..., F, N, d_k]   v, out [..., F, N, d_v]
    beta  [..., F, N] fp32   gate   [...] fp32
q, k, v, out are torch.bfloat16 (vda_forward) or torch.float32
(vda_forward_f32), contiguous, on one GPU.
"""
from __future__ import annotations

import ctypes
import math
import os
import re

# torch is imported before libvda.so is loaded: torch bundles its own HIP
# runtime (soname libamdhip64.so.7), and loading it first makes libvda.so's
# dependency resolve to that same runtime, so torch's streams and memory are
# valid in the library's calls.  Loading libvda.so first would bring in a
# second runtime instance whose streams are unrelated to torch's.
import torch  # noqa: F401  (load order matters, see above)

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libvda.so")
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "vda.h")

VDA_OK = 0
STATUS_NAMES = {0: "VDA_OK", 1: "VDA_ERR_NULL", 2: "VDA_ERR_SIZE", 3: "VDA_ERR_UNSUPPORTED",
                4: "VDA_ERR_ALIGN", 5: "VDA_ERR_OVERLAP", 6: "VDA_ERR_HIP", 7: "VDA_ERR_NOMEM",
                8: "VDA_ERR_SCRATCH"}

_P = ctypes.c_void_p
_I = ctypes.c_int

class VdaOptions(ctypes.Structure):
    """struct vda_options (include/vda.h)."""
    _fields_ = [("rule", ctypes.c_int), ("alpha", ctypes.c_void_p),
                ("text_state", ctypes.c_void_p), ("window_chunk", ctypes.c_int),
                ("window_radius", ctypes.c_int), ("window_offset", ctypes.c_int),
                ("gate_tokens", ctypes.c_void_p), ("out_heads", ctypes.c_int),
                ("q_heads", ctypes.c_int)]


class VdaDeltaProblem(ctypes.Structure):
    """struct vda_delta_problem (include/vda.h)."""
    _fields_ = [("T", ctypes.c_int), ("n_seqs", ctypes.c_int), ("cu_seqlens", ctypes.c_void_p),
                ("H_k", ctypes.c_int), ("H_v", ctypes.c_int), ("d_k", ctypes.c_int),
                ("d_v", ctypes.c_int), ("layout", ctypes.c_int), ("is_f32", ctypes.c_int),
                ("scale", ctypes.c_float)]


class VdaRopeOptions(ctypes.Structure):
    """struct vda_rope_options (include/vda.h)."""
    _fields_ = [(n, ctypes.c_int) for n in (
        "pairs_t", "pairs_h", "pairs_w", "interleaved", "l2", "layout", "grid_h", "grid_w",
        "frame_offset", "x_row_stride", "dx_row_stride")]


RULES = {"joint": 0, "frozen": 1}
LAYOUTS = {"heads": 0, "tokens": 1}

_SIGNATURES = {
    "vda_status_string": (ctypes.c_char_p, [_I]),
    "vda_forward": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P]),
    "vda_forward_f32": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P]),
    "vda_forward_noalloc": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P]),
    "vda_forward_ex": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "vda_forward_ex_f32": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "vda_text_state": (_I, [_P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P]),
    "vda_default_split_plan": (_I, [_I, _I, _I, _I, _I, _I, _P, _P]),
    "vda_frame_stats": (_I, [_P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P, _P, _P]),
    "vda_frame_inverse": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P]),
    "vda_frame_inverse_tiles": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P]),
    "vda_state_scan": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "vda_state_scan_tiles": (_I, [_P, _P, _I, _I, _I, _I, _P, _P, _P]),
    "vda_state_scan_chunked": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P]),
    "vda_state_scan_chunked_workspace": (ctypes.c_size_t, [_I, _I, _I, _I, _I, _I]),
    "vda_prep": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P]),
    "vda_readout": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P]),
    "vda_delta_forward": (_I, [_P] * 11),
    "vda_delta_forward_workspace": (ctypes.c_size_t, [_P]),
    "vda_delta_backward": (_I, [_P] * 17),
    "vda_delta_backward_workspace": (ctypes.c_size_t, [_P]),
    "vda_delta_step": (_I, [_P] * 5 + [_I] * 7 + [ctypes.c_float, _P, _I, _P, _P, _P]),
    "vda_rope": (_I, [_P, _P, _P, _I, _I, _I, _I, _P, _I, _P, _P]),
    "vda_rope_backward": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _P, _I, _P, _P]),
    "vda_release_workspace": (_I, [_I, _P]),
    "vda_workspace_bytes": (_I, [_I, _P]),
}


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2609_20744_amd.build` "
            "(the VDA operator has no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


class VDAError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def status_string(status: int) -> str:
    return lib.vda_status_string(int(status)).decode()


def header_functions() -> list[str]:
    """Names of the entry points declared in include/vda.h."""
    with open(HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?(vda_\w+)\s*\(", text, flags=re.M)))


def _check(status: int, where: str) -> None:
    if status != VDA_OK:
        if status == 1:
            raise ValueError(f"{where}: {status_string(status)}")
        if status in (2, 3, 4, 5, 8):
            raise ValueError(f"{where}: {status_string(status)}")
        raise VDAError(status, where)


# ----------------------------------------------------------------------------
# torch-facing wrappers
# ----------------------------------------------------------------------------

def _torch():
    return torch


# The raw handle of a device's current stream without a Stream object around
# it (about 1 us a call); the public spelling where torch lacks it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(device, stream=None) -> int:
    if device.type != "cuda":
        torch.cuda.device(device)  # raises: not a cuda device
    if stream is not None:
        return int(stream.cuda_stream)
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return int(torch.cuda.current_stream(device).cuda_stream)


def _call(fn, device, *args) -> int:
    """fn(*args) with `device` current; switching is left out where it is."""
    if device.index == torch.cuda.current_device():
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _require(t, name, dtype, device):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device
            and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _shape(q, k, v, beta, gate=None, q_heads=0):
    if k.dim() < 3:
        raise ValueError("k must be [..., F, N, d_k]")
    lead = tuple(k.shape[:-3])
    F, N, d_k = k.shape[-3:]
    d_v = v.shape[-1]
    H = math.prod(lead) if lead else 1
    if q_heads:
        if H % q_heads:
            raise ValueError(f"q_heads {q_heads} must divide the {H} head problems")
        qshape = (H // q_heads, F, N, q_heads * d_k)
        if tuple(q.shape) != qshape:
            raise ValueError(f"raw q shape {tuple(q.shape)} must be {qshape}")
    elif tuple(k.shape) != tuple(q.shape):
        raise ValueError(f"k shape {tuple(k.shape)} != q shape {tuple(q.shape)}")
    if tuple(v.shape) != lead + (F, N, d_v):
        raise ValueError(f"v shape {tuple(v.shape)} does not match k")
    if tuple(beta.shape) != lead + (F, N):
        raise ValueError(f"beta shape {tuple(beta.shape)} must be {lead + (F, N)}")
    if gate is not None and gate.numel() != H:
        raise ValueError(f"gate must have {H} elements (one per head problem)")
    return lead, F, N, H, d_k, d_v


def forward(q, k, v, beta, gate, out=None, stream=None, alpha=None, text_state=None,
            window=None, rule="joint", gate_tokens=None, out_heads=None, q_heads=None):
    """VDA forward (vda_forward for bf16 tensors, vda_forward_f32 for fp32).

    With any of the full-operator options it calls vda_forward_ex(_f32):
    alpha [..., F, d_k] fp32 channel decays, text_state [..., d_v, d_k] fp32
    S_T, window = (chunk, radius, offset) of the local window, rule 'joint'
    (Eq. 5) or 'frozen' (Eq. 3c with 1/sqrt(U) key scaling), and
    gate_tokens [..., F, N, d_v] (q's dtype), the output gate G^L of Eq. 1c
    per token and channel, which replaces the per-head gate (gate may then
    be None).  out_heads (> 0) selects the token-major output
    [H / out_heads, F, N, out_heads * d_v] of clips of out_heads heads, H the
    number of head problems (the product of the leading dimensions).
    q_heads (> 0) passes the raw token-major query [H / q_heads, F, N,
    q_heads * d_k] (as vda_prep's input) and leaves its L2 map to the
    readout; k, v and the other arguments keep their per-head layouts."""
    torch = _torch()
    dt = q.dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise ValueError(f"q dtype {dt} must be bfloat16 or float32")
    dev = q.device
    if dev.type != "cuda":
        raise ValueError("VDA runs on the GPU only; tensors must be on a cuda device")
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, n, dt, dev)
    _require(beta, "beta", torch.float32, dev)
    if gate is not None or gate_tokens is None:
        _require(gate, "gate", torch.float32, dev)
    qh = int(q_heads or 0)
    if qh < 0:
        raise ValueError(f"q_heads {q_heads} must be positive")
    lead, F, N, H, d_k, d_v = _shape(q, k, v, beta, gate, qh)
    oh = int(out_heads or 0)
    if oh < 0 or (oh and H % oh):
        raise ValueError(f"out_heads {out_heads} must divide the {H} head problems")
    oshape = (H // oh, F, N, oh * d_v) if oh else lead + (F, N, d_v)
    if out is None:
        out = torch.empty(oshape, dtype=dt, device=dev)
    else:
        _require(out, "out", dt, dev)
        if tuple(out.shape) != oshape:
            raise ValueError(f"out shape {tuple(out.shape)} must be {oshape}")
    if alpha is None and text_state is None and window is None and rule == "joint" and \
            gate_tokens is None and not oh and not qh:
        fn = lib.vda_forward if dt == torch.bfloat16 else lib.vda_forward_f32
        st = _call(fn, dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
                   gate.data_ptr(), F, N, H, d_k, d_v, out.data_ptr(), _stream_ptr(dev, stream))
        _check(st, fn.__name__)
        return out
    if rule not in RULES:
        raise ValueError(f"rule must be one of {sorted(RULES)}")
    if alpha is not None:
        _require(alpha, "alpha", torch.float32, dev)
        if tuple(alpha.shape) != lead + (F, d_k):
            raise ValueError(f"alpha shape {tuple(alpha.shape)} must be {lead + (F, d_k)}")
    if text_state is not None:
        _require(text_state, "text_state", torch.float32, dev)
        if tuple(text_state.shape) != lead + (d_v, d_k):
            raise ValueError(f"text_state shape {tuple(text_state.shape)} must be "
                             f"{lead + (d_v, d_k)}")
    if gate_tokens is not None:
        _require(gate_tokens, "gate_tokens", dt, dev)
        if tuple(gate_tokens.shape) != lead + (F, N, d_v):
            raise ValueError(f"gate_tokens shape {tuple(gate_tokens.shape)} must be "
                             f"{lead + (F, N, d_v)}")
    chunk, radius, offset = (1, 0, 0) if window is None else (int(x) for x in window)
    opts = VdaOptions(RULES[rule], alpha.data_ptr() if alpha is not None else None,
                      text_state.data_ptr() if text_state is not None else None,
                      chunk, radius, offset,
                      gate_tokens.data_ptr() if gate_tokens is not None else None, oh, qh)
    fn = lib.vda_forward_ex if dt == torch.bfloat16 else lib.vda_forward_ex_f32
    st = _call(fn, dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(),
               gate.data_ptr() if gate is not None else None, F, N, H, d_k, d_v,
               ctypes.byref(opts), out.data_ptr(), _stream_ptr(dev, stream))
    _check(st, fn.__name__)
    return out


def text_state(k, v, beta, rule="joint", out=None, stream=None):
    """The prompt state S_T (vda_text_state): k [..., L, d_k], v [..., L, d_v]
    (bfloat16 or float32), beta [..., L] float32; returns [..., d_v, d_k]
    float32, the text_state argument of forward."""
    torch = _torch()
    dt = k.dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise ValueError(f"k dtype {dt} must be bfloat16 or float32")
    dev = k.device
    if dev.type != "cuda":
        raise ValueError("VDA runs on the GPU only; tensors must be on a cuda device")
    _require(k, "k", dt, dev)
    _require(v, "v", dt, dev)
    _require(beta, "beta", torch.float32, dev)
    if rule not in RULES:
        raise ValueError(f"rule must be one of {sorted(RULES)}")
    if k.dim() < 2:
        raise ValueError("k must be [..., L, d_k]")
    lead = tuple(k.shape[:-2])
    L, d_k = k.shape[-2:]
    d_v = v.shape[-1]
    H = math.prod(lead) if lead else 1
    if tuple(v.shape) != lead + (L, d_v):
        raise ValueError(f"v shape {tuple(v.shape)} does not match k")
    if tuple(beta.shape) != lead + (L,):
        raise ValueError(f"beta shape {tuple(beta.shape)} must be {lead + (L,)}")
    if out is None:
        out = torch.empty(lead + (d_v, d_k), dtype=torch.float32, device=dev)
    else:
        _require(out, "out", torch.float32, dev)
        if tuple(out.shape) != lead + (d_v, d_k):
            raise ValueError(f"out shape {tuple(out.shape)} must be {lead + (d_v, d_k)}")
    st = _call(lib.vda_text_state, dev, k.data_ptr(), v.data_ptr(), beta.data_ptr(), L, H, d_k,
               d_v, RULES[rule], int(dt == torch.float32), out.data_ptr(),
               _stream_ptr(dev, stream))
    _check(st, "vda_text_state")
    return out


def forward_noalloc(q, k, v, beta, gate, out=None, stream=None):
    """vda_forward_noalloc: vda_forward (bf16 tensors) with the library's
    fixed device scratch array as workspace; the library allocates nothing
    (out is allocated here by torch when not given)."""
    torch = _torch()
    dev = q.device
    if q.dtype != torch.bfloat16:
        raise ValueError("vda_forward_noalloc takes bfloat16 q, k, v")
    if dev.type != "cuda":
        raise ValueError("VDA runs on the GPU only; tensors must be on a cuda device")
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, n, torch.bfloat16, dev)
    _require(beta, "beta", torch.float32, dev)
    _require(gate, "gate", torch.float32, dev)
    lead, F, N, H, d_k, d_v = _shape(q, k, v, beta, gate)
    if out is None:
        out = torch.empty(lead + (F, N, d_v), dtype=q.dtype, device=dev)
    else:
        _require(out, "out", q.dtype, dev)
        if tuple(out.shape) != lead + (F, N, d_v):
            raise ValueError(f"out shape {tuple(out.shape)} must be {lead + (F, N, d_v)}")
    st = _call(lib.vda_forward_noalloc, dev, q.data_ptr(), k.data_ptr(), v.data_ptr(),
               beta.data_ptr(), gate.data_ptr(), F, N, H, d_k, d_v, out.data_ptr(),
               _stream_ptr(dev, stream))
    _check(st, "vda_forward_noalloc")
    return out


def release_workspace(device: int = -1) -> int:
    """Free the library's cached workspace buffers on `device` (-1: the
    current one) that no call is using (vda_release_workspace); waits for
    their last work on the host.  Returns the bytes freed."""
    n = ctypes.c_size_t(0)
    _check(lib.vda_release_workspace(int(device), ctypes.byref(n)), "vda_release_workspace")
    return n.value


def workspace_bytes(device: int = -1) -> int:
    """Bytes of workspace the library holds cached on `device` (-1: the
    current one) (vda_workspace_bytes)."""
    n = ctypes.c_size_t(0)
    _check(lib.vda_workspace_bytes(int(device), ctypes.byref(n)), "vda_workspace_bytes")
    return n.value


def default_split_plan(F: int, N: int, H: int, d_k: int, d_v: int,
                       is_f32: bool = False) -> tuple[int, int]:
    """(tail_frames, splits) of the statistics step that vda_forward uses on
    the current device (vda_default_split_plan)."""
    t, s = ctypes.c_int(0), ctypes.c_int(0)
    st = lib.vda_default_split_plan(F, N, H, d_k, d_v, int(bool(is_f32)), ctypes.byref(t),
                                    ctypes.byref(s))
    _check(st, "vda_default_split_plan")
    return t.value, s.value


def partial_count(count: int, tail_frames: int, splits: int) -> int:
    """Number of partial matrices of a split plan over `count` frames."""
    return count + tail_frames * (splits - 1) if splits > 1 else count


def frame_stats(k, v, beta, splits=None, tail_frames=None, A_part=None, B_part=None,
                stream=None):
    """Step a1 (vda_frame_stats): partial A [P, d_k, d_k] and B [P, d_v, d_k],
    fp32, under the split plan (tail_frames, splits); the first H*F partials
    are the frames in [H, F] order.  Defaults: the library's plan; with only
    `splits` given, every frame is split."""
    torch = _torch()
    dev, dt = k.device, k.dtype
    for t, n in ((k, "k"), (v, "v")):
        _require(t, n, dt, dev)
    _require(beta, "beta", torch.float32, dev)
    lead, F, N, H, d_k, d_v = _shape(k, k, v, beta)
    if splits is None:
        with torch.cuda.device(dev):
            tail_frames, splits = default_split_plan(F, N, H, d_k, d_v, dt == torch.float32)
    elif tail_frames is None:
        tail_frames = H * F
    splits, tail_frames = int(splits), int(tail_frames)
    P = partial_count(H * F, tail_frames, splits)
    if A_part is None:
        A_part = torch.empty((P, d_k, d_k), dtype=torch.float32, device=dev)
    if B_part is None:
        B_part = torch.empty((P, d_v, d_k), dtype=torch.float32, device=dev)
    st = _call(lib.vda_frame_stats, dev, k.data_ptr(), v.data_ptr(), beta.data_ptr(), F, N, H, d_k,
               d_v, tail_frames, splits, int(dt == torch.float32), A_part.data_ptr(),
               B_part.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_frame_stats")
    return A_part, B_part


def frame_inverse(A_part, B_part=None, count=None, tail_frames=0, splits=1, Inv=None,
                  stream=None, tiles=False):
    """Step a2 (vda_frame_inverse): Inv [count, d_k, d_k] = (I + sum of each
    frame's A partials)^-1, fp32, under the split plan that made the partials
    (A_part [P, d_k, d_k]; count defaults to P when splits == 1).  With
    splits > 1 each frame's B partials ([P, d_v, d_k]) are folded in place into
    B_part[frame].  tiles=True (vda_frame_inverse_tiles) writes each inverse
    as split-bf16 operand tiles instead: Inv is then [count, 2, d_k * d_k]
    bfloat16 (hi plane, lo plane; the layout of include/vda.h), or any
    buffer of the same size in bytes."""
    torch = _torch()
    d_k = A_part.shape[-1]
    if count is None:
        if splits > 1:
            raise ValueError("count is required with a split plan")
        count = math.prod(A_part.shape[:-2])
    d_v = B_part.shape[-2] if B_part is not None else d_k
    if splits > 1 and B_part is None:
        raise ValueError("B_part is required when there is more than one split")
    if Inv is None:
        Inv = (torch.empty((count, 2, d_k * d_k), dtype=torch.bfloat16, device=A_part.device)
               if tiles else
               torch.empty((count, d_k, d_k), dtype=torch.float32, device=A_part.device))
    fn = lib.vda_frame_inverse_tiles if tiles else lib.vda_frame_inverse
    st = _call(fn, A_part.device, A_part.data_ptr(),
               B_part.data_ptr() if B_part is not None else None, int(tail_frames), int(splits),
               int(count), d_k, d_v, Inv.data_ptr(), _stream_ptr(A_part.device, stream))
    _check(st, fn.__name__)
    return Inv


def state_scan(Inv, B, S_fwd=None, S_rev=None, exact_f32=False, stream=None):
    """Steps a3/a4 (vda_state_scan).  Inv [H, F, d_k, d_k], B [H, F, d_v, d_k]
    (the reduced statistic, e.g. B_part[0] after frame_inverse).
    exact_f32 selects fp32 matrix products (the fp32 storage path); otherwise
    split-bf16 products with fp32 accumulation (the bf16 storage path)."""
    torch = _torch()
    H, F, d_v, d_k = B.shape
    dev = B.device
    if S_fwd is None:
        S_fwd = torch.empty((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    if S_rev is None:
        S_rev = torch.empty((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    st = _call(lib.vda_state_scan, dev, Inv.data_ptr(), B.data_ptr(), F, H, d_k, d_v,
               int(bool(exact_f32)), S_fwd.data_ptr(), S_rev.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_state_scan")
    return S_fwd, S_rev


def state_scan_tiles(Inv_tiles, B, S_fwd=None, S_rev=None, stream=None):
    """Steps a3/a4 from split-bf16 operand tiles (vda_state_scan_tiles), the
    kernel vda_forward runs with bf16 storage.  Inv_tiles: [H, F, ...] with
    d_k * d_k * 4 bytes per frame (as written by frame_inverse(tiles=True));
    B [H, F, d_v, d_k] fp32."""
    torch = _torch()
    H, F, d_v, d_k = B.shape
    dev = B.device
    if Inv_tiles.numel() * Inv_tiles.element_size() != H * F * d_k * d_k * 4:
        raise ValueError("Inv_tiles must hold d_k * d_k * 4 bytes per frame")
    if S_fwd is None:
        S_fwd = torch.empty((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    if S_rev is None:
        S_rev = torch.empty((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    st = _call(lib.vda_state_scan_tiles, dev, Inv_tiles.data_ptr(), B.data_ptr(), F, H, d_k, d_v,
               S_fwd.data_ptr(), S_rev.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_state_scan_tiles")
    return S_fwd, S_rev


def state_scan_chunked(Inv_tiles, B, chunk, offset=0, alpha=None, text_state=None, S_fwd=None,
                       S_rev=None, work=None, stream=None):
    """Chunk-wise scans for a chunked window (vda_state_scan_chunked): the
    states entering every chunk of the window grid, forward at the chunk's
    first frame of S_fwd, reverse at its last frame of S_rev (other frames
    untouched; new outputs are zero-filled).  Inv_tiles as for
    state_scan_tiles, B [H, F, d_v, d_k] fp32, alpha [H, F, d_k] and
    text_state [H, d_v, d_k] fp32 or None; work: a device buffer of
    chunked_workspace(...) bytes (allocated if None)."""
    torch = _torch()
    H, F, d_v, d_k = B.shape
    dev = B.device
    if Inv_tiles.numel() * Inv_tiles.element_size() != H * F * d_k * d_k * 4:
        raise ValueError("Inv_tiles must hold d_k * d_k * 4 bytes per frame")
    for t, n in ((alpha, "alpha"), (text_state, "text_state")):
        if t is not None:
            _require(t, n, torch.float32, dev)
    if S_fwd is None:
        S_fwd = torch.zeros((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    if S_rev is None:
        S_rev = torch.zeros((H, F, d_v, d_k), dtype=torch.float32, device=dev)
    if work is None:
        nbytes = chunked_workspace(F, H, d_k, d_v, chunk, offset)
        work = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)
    st = _call(lib.vda_state_scan_chunked, dev, Inv_tiles.data_ptr(), B.data_ptr(),
               alpha.data_ptr() if alpha is not None else None,
               text_state.data_ptr() if text_state is not None else None, F, H, d_k, d_v,
               int(chunk), int(offset), work.data_ptr(), S_fwd.data_ptr(), S_rev.data_ptr(),
               _stream_ptr(dev, stream))
    _check(st, "vda_state_scan_chunked")
    return S_fwd, S_rev


def chunked_workspace(F: int, H: int, d_k: int, d_v: int, chunk: int, offset: int = 0) -> int:
    """Bytes of the work buffer of state_scan_chunked."""
    return int(lib.vda_state_scan_chunked_workspace(F, H, d_k, d_v, int(chunk), int(offset)))


def prep(q, k, v, grid, wk_spatial, wk_temporal, wv_spatial, wv_temporal, H, outs=None,
         stream=None):
    """VDA-Prep (vda_prep): q, k [B, F, N, H*d_k], v [B, F, N, H*d_v] bf16
    projections with N = grid[0] * grid[1]; filters fp32 wk_spatial
    [H*d_k, 25] (or [H*d_k, 5, 5]), wk_temporal [H*d_k, 5], likewise for v.
    Returns (q', k', v') [B*H, F, N, d] bf16 (or fills `outs`).  With q None
    the query map is skipped (forward with q_heads = H applies it to the raw
    query) and q' is None."""
    torch = _torch()
    dev = k.device
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        if t is not None or n != "q":
            _require(t, n, torch.bfloat16, dev)
    for t, n in ((wk_spatial, "wk_spatial"), (wk_temporal, "wk_temporal"),
                 (wv_spatial, "wv_spatial"), (wv_temporal, "wv_temporal")):
        _require(t, n, torch.float32, dev)
    B, F, N, Ck = k.shape
    Cv = v.shape[-1]
    gh, gw = grid
    if gh * gw != N or (q is not None and q.shape != k.shape) or v.shape[:3] != k.shape[:3]:
        raise ValueError("q, k, v must be [B, F, grid_h*grid_w, H*d]")
    if Ck % H or Cv % H:
        raise ValueError("channels must split into H heads")
    d_k, d_v = Ck // H, Cv // H
    if outs is None:
        outs = (torch.empty((B * H, F, N, d_k), dtype=torch.bfloat16, device=dev)
                if q is not None else None,
                torch.empty((B * H, F, N, d_k), dtype=torch.bfloat16, device=dev),
                torch.empty((B * H, F, N, d_v), dtype=torch.bfloat16, device=dev))
    elif (outs[0] is None) != (q is None):
        raise ValueError("q and its output must both be given or both be None")
    st = _call(lib.vda_prep, dev, q.data_ptr() if q is not None else None, k.data_ptr(),
               v.data_ptr(), wk_spatial.data_ptr(), wk_temporal.data_ptr(), wv_spatial.data_ptr(),
               wv_temporal.data_ptr(), B, F, gh, gw, H, d_k, d_v,
               outs[0].data_ptr() if outs[0] is not None else None, outs[1].data_ptr(),
               outs[2].data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_prep")
    return outs


def readout(q, S_fwd, S_rev, gate, d_v=None, out=None, stream=None):
    """Steps a5-a7 (vda_readout).  q [H, F, N, d_k], S_* [H, F, d_v, d_k], gate [H]."""
    torch = _torch()
    H, F, N, d_k = q.shape
    d_v = S_fwd.shape[-2] if d_v is None else d_v
    dev = q.device
    if out is None:
        out = torch.empty((H, F, N, d_v), dtype=q.dtype, device=dev)
    st = _call(lib.vda_readout, dev, q.data_ptr(), S_fwd.data_ptr(), S_rev.data_ptr(),
               gate.data_ptr(), F, N, H, d_k, d_v, int(q.dtype == torch.float32), out.data_ptr(),
               _stream_ptr(dev, stream))
    _check(st, "vda_readout")
    return out


# ----------------------------------------------------------------------------
# The token-wise gated delta rule and rotary positions
# ----------------------------------------------------------------------------

def _ptr(t):
    return t.data_ptr() if t is not None else None


def _new(shape, dtype, dev, stream):
    """An empty tensor that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


def _expect(t, name, shape, dtype, dev):
    _require(t, name, dtype, dev)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} shape {tuple(t.shape)} must be {tuple(shape)}")


def _storage(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{name} dtype {t.dtype} must be bfloat16 or float32")
    if t.device.type != "cuda":
        raise ValueError("VDA runs on the GPU only; tensors must be on a cuda device")
    return t.dtype, t.device


def _delta_problem(q, k, v, g, beta, cu_seqlens, layout, scale):
    """The problem, and the shape of its states."""
    dt, dev = _storage(q, "q")
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, n, dt, dev)
    _require(g, "g", torch.float32, dev)
    _require(beta, "beta", torch.float32, dev)
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    if q.dim() < 3 or v.dim() != q.dim():
        raise ValueError("q, k, v must be [..., H, L, d] (heads) or [..., L, H, d] (tokens)")
    if k.shape != q.shape:
        raise ValueError(f"k shape {tuple(k.shape)} != q shape {tuple(q.shape)}")
    lead, heads = tuple(q.shape[:-3]), layout == "heads"
    H_k, L = (q.shape[-3], q.shape[-2]) if heads else (q.shape[-2], q.shape[-3])
    H_v = v.shape[-3] if heads else v.shape[-2]
    d_k, d_v = q.shape[-1], v.shape[-1]
    gates = lead + ((H_v, L) if heads else (L, H_v))
    if tuple(v.shape) != gates + (d_v,):
        raise ValueError(f"v shape {tuple(v.shape)} does not match q")
    for t, n in ((g, "g"), (beta, "beta")):
        if tuple(t.shape) != gates:
            raise ValueError(f"{n} shape {tuple(t.shape)} must be {gates}")
    if H_k < 1 or H_v % H_k:
        raise ValueError(f"{H_v} value heads must be a multiple of {H_k} key heads")
    B = math.prod(lead)
    if cu_seqlens is not None:
        if lead:
            raise ValueError("with cu_seqlens, q, k, v have three dimensions (one packed batch)")
        _require(cu_seqlens, "cu_seqlens", torch.int32, dev)
        if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
            raise ValueError("cu_seqlens must hold one more offset than there are sequences")
        n, states = cu_seqlens.numel() - 1, (cu_seqlens.numel() - 1, H_v, d_v, d_k)
        T, Hk, Hv = L, H_k, H_v
    elif heads:  # every leading index and head is a head problem of its own
        n, T, Hk, Hv = 1, L, B * H_k, B * H_v
        states = lead + (H_v, d_v, d_k)
    else:
        n, T, Hk, Hv = B, B * L, H_k, H_v
        states = lead + (H_v, d_v, d_k)
    p = VdaDeltaProblem(T, n, _ptr(cu_seqlens), Hk, Hv, d_k, d_v, LAYOUTS[layout],
                        int(dt == torch.float32), 1.0 if scale is None else float(scale))
    return p, states, dt, dev


def _delta_workspace(fn, p, dev, stream):
    nbytes = _call(fn, dev, ctypes.byref(p))
    return _new((max(int(nbytes), 16),), torch.uint8, dev, stream)


def delta_forward(q, k, v, g, beta, cu_seqlens=None, layout="heads", scale=None, state=None,
                  return_state=False, out=None, state_out=None, work=None, stream=None):
    """The token-wise gated delta rule over whole sequences (vda_delta_forward).

    layout 'heads': q, k [..., H_k, L, d_k], v [..., H_v, L, d_v], g, beta
    [..., H_v, L]; 'tokens': q, k [..., L, H_k, d_k], v [..., L, H_v, d_v], g,
    beta [..., L, H_v]; H_v a multiple of H_k; q, k, v bfloat16 or float32,
    g (log decay) and beta float32.  Each leading index is a sequence; with
    cu_seqlens (int32 [n + 1]) there is none, and the L tokens are n packed
    sequences.  state: the states to start from, [..., H_v, d_v, d_k] float32
    ([n, H_v, d_v, d_k] with cu_seqlens), or None (zero).  scale defaults to 1.
    Returns the output (v's shape), or (output, last states) with
    return_state.  work: a device buffer of delta_workspace(...) bytes
    (allocated if None); calls that may run at the same time need their own.
    Packed rows outside every sequence are left as they are in `out` (a new
    output holds anything there).  Nothing is recorded for autograd: the
    gradients come from delta_backward."""
    p, states, dt, dev = _delta_problem(q, k, v, g, beta, cu_seqlens, layout, scale)
    if state is not None:
        _expect(state, "state", states, torch.float32, dev)
    if out is None:
        out = _new(v.shape, dt, dev, stream)
    else:
        _expect(out, "out", v.shape, dt, dev)
    if state_out is not None:
        _expect(state_out, "state_out", states, torch.float32, dev)
    elif return_state:
        state_out = _new(states, torch.float32, dev, stream)
    if work is None:
        work = _delta_workspace(lib.vda_delta_forward_workspace, p, dev, stream)
    else:
        _delta_work(work, p, lib.vda_delta_forward_workspace, dev)
    st = _call(lib.vda_delta_forward, dev, ctypes.byref(p), q.data_ptr(), k.data_ptr(),
               v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state), out.data_ptr(),
               _ptr(state_out), work.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_delta_forward")
    return (out, state_out) if return_state else out


def _delta_work(work, p, fn, dev):
    _require(work, "work", torch.uint8, dev)
    need = int(_call(fn, dev, ctypes.byref(p)))
    if work.numel() < need:
        raise ValueError(f"work holds {work.numel()} bytes, {need} are needed")


def delta_workspace(q, k, v, g, beta, cu_seqlens=None, layout="heads", backward=False):
    """Bytes of the work buffer of delta_forward (or delta_backward) for these arguments."""
    p, _, _, dev = _delta_problem(q, k, v, g, beta, cu_seqlens, layout, None)
    fn = lib.vda_delta_backward_workspace if backward else lib.vda_delta_forward_workspace
    return int(_call(fn, dev, ctypes.byref(p)))


def delta_backward(dout, q, k, v, g, beta, cu_seqlens=None, layout="heads", scale=None, state=None,
                   dstate=None, outs=None, work=None, stream=None):
    """The gradients of delta_forward (vda_delta_backward): dout of the
    output, dstate of the last states (or None: zero); the other arguments as
    there.  Returns (dq, dk, dv, dg, dbeta, dstate_in), dstate_in None where
    state is None; `outs`, such a tuple, is filled instead of new tensors."""
    p, states, dt, dev = _delta_problem(q, k, v, g, beta, cu_seqlens, layout, scale)
    _expect(dout, "dout", v.shape, dt, dev)
    for t, n in ((state, "state"), (dstate, "dstate")):
        if t is not None:
            _expect(t, n, states, torch.float32, dev)
    shapes = ((q.shape, dt), (k.shape, dt), (v.shape, dt), (g.shape, torch.float32),
              (beta.shape, torch.float32), (states, torch.float32))
    names = ("dq", "dk", "dv", "dg", "dbeta", "dstate_in")
    if outs is None:
        outs = tuple(_new(s, d, dev, stream) if n != "dstate_in" or state is not None else None
                     for n, (s, d) in zip(names, shapes))
    else:
        if len(outs) != 6:
            raise ValueError("outs must be (dq, dk, dv, dg, dbeta, dstate_in)")
        for t, n, (s, d) in zip(outs, names, shapes):
            if t is not None or n != "dstate_in":
                _expect(t, n, s, d, dev)
    if work is None:
        work = _delta_workspace(lib.vda_delta_backward_workspace, p, dev, stream)
    else:
        _delta_work(work, p, lib.vda_delta_backward_workspace, dev)
    st = _call(lib.vda_delta_backward, dev, ctypes.byref(p), dout.data_ptr(), q.data_ptr(),
               k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state),
               _ptr(dstate), *(_ptr(t) for t in outs), work.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_delta_backward")
    return tuple(outs)


def delta_step(q, k, v, g, beta, state, slots=None, scale=None, out=None, stream=None):
    """A few tokens of each of n sequences (vda_delta_step): q, k [n, t, H_k,
    d_k], v [n, t, H_v, d_v] bfloat16 or float32, g, beta [n, t, H_v]
    float32; state [n_slots, H_v, d_v, d_k] float32, updated in place.  slots:
    int32 [n], the sequences' slots (distinct; one outside the pool marks a
    row of padding, whose output is left as it is), or None (slot i for
    sequence i).  Returns the output [n, t, H_v, d_v]."""
    dt, dev = _storage(q, "q")
    if q.dim() != 4 or not isinstance(v, torch.Tensor) or v.dim() != 4:
        raise ValueError("q, k must be [n, t, H_k, d_k] and v [n, t, H_v, d_v]")
    n, t, H_k, d_k = q.shape
    H_v, d_v = v.shape[2:]
    _require(q, "q", dt, dev)
    _expect(k, "k", q.shape, dt, dev)
    _expect(v, "v", (n, t, H_v, d_v), dt, dev)
    _expect(g, "g", (n, t, H_v), torch.float32, dev)
    _expect(beta, "beta", (n, t, H_v), torch.float32, dev)
    _require(state, "state", torch.float32, dev)
    if state.dim() != 4 or tuple(state.shape[1:]) != (H_v, d_v, d_k):
        raise ValueError(f"state shape {tuple(state.shape)} must be [n_slots, {H_v}, {d_v}, {d_k}]")
    if slots is not None:
        _expect(slots, "slots", (n,), torch.int32, dev)
    if out is None:
        out = _new(v.shape, dt, dev, stream)
    else:
        _expect(out, "out", v.shape, dt, dev)
    st = _call(lib.vda_delta_step, dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(),
               beta.data_ptr(), n, t, H_k, H_v, d_k, d_v, int(dt == torch.float32),
               1.0 if scale is None else float(scale), _ptr(slots), state.shape[0],
               state.data_ptr(), out.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_delta_step")
    return out


def _int32(name, x):
    """x as an int that a C int holds; ctypes would take it modulo 2^32."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} {x} does not fit 32 bits")
    return x


def _token_rows(t, name, H):
    """Row stride of a [B, L, H * d] tensor whose token rows are equally far apart."""
    if H < 1 or t.dim() != 3 or t.shape[2] % H:
        raise ValueError(f"{name} must be [B, L, H * d], H at least 1")
    B, L, C = t.shape
    row = t.stride(1) if L > 1 else t.stride(0) if B > 1 else C
    if t.stride(2) != 1 or row < C or (B > 1 and t.stride(0) != L * row):
        raise ValueError(f"{name} must have contiguous rows at one stride over the batch and tokens")
    return _int32(f"the row stride of {name}", row)


def _rope_args(inv_freq, axes, H, B, L, d, positions, grid, frame_offset, interleaved, l2, layout,
               dev):
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    pt, ph, pw = (_int32("axes", a) for a in axes)
    for n, x in (("H", H), ("B", B), ("L", L)):
        _int32(n, x)
    _expect(inv_freq, "inv_freq", (pt + ph + pw,), torch.float32, dev)
    if positions is not None:
        if grid is not None:
            raise ValueError("give positions or a grid, not both")
        _expect(positions, "positions", (B, L, 3), torch.int32, dev)
        gh = gw = 1
    elif grid is None:
        raise ValueError("positions or a grid (height, width) is needed")
    else:
        gh, gw = (_int32("grid", x) for x in grid)
    return VdaRopeOptions(pt, ph, pw, int(bool(interleaved)), int(bool(l2)), LAYOUTS[layout], gh, gw,
                          _int32("frame_offset", frame_offset), 0, 0)


def rope(x, inv_freq, axes, H, positions=None, grid=None, frame_offset=0, interleaved=True,
         l2=False, layout="heads", out=None, stream=None):
    """Rotary positions over time, height and width (vda_rope): x [B, L, H*d]
    bfloat16 or float32 (a slice of a fused projection's channels is fine),
    axes = (pairs of time, of height, of width), inv_freq float32 [sum of
    axes].  The tokens' positions: `positions` int32 [B, L, 3], or grid =
    (height, width) with the first frame at frame_offset.  l2 divides each
    token of each head by its length first.  Returns [B * H, L, d] (layout
    'heads', as prep) or [B, L, H * d] ('tokens').  Nothing is recorded for
    autograd: the gradient comes from rope_backward."""
    dt, dev = _storage(x, "x")
    row = _token_rows(x, "x", H)
    B, L, C = x.shape
    d = C // H
    o = _rope_args(inv_freq, axes, H, B, L, d, positions, grid, frame_offset, interleaved, l2,
                   layout, dev)
    o.x_row_stride = row
    shape = (B * H, L, d) if layout == "heads" else (B, L, C)
    if out is None:
        out = _new(shape, dt, dev, stream)
    else:
        _expect(out, "out", shape, dt, dev)
    st = _call(lib.vda_rope, dev, x.data_ptr(), inv_freq.data_ptr(), _ptr(positions), B, L, H, d,
               ctypes.byref(o), int(dt == torch.float32), out.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_rope")
    return out


def rope_backward(dout, inv_freq, axes, H, x=None, positions=None, grid=None, frame_offset=0,
                  interleaved=True, l2=False, layout="heads", out=None, stream=None):
    """The gradient of rope (vda_rope_backward): dout in the output's layout,
    x the forward input (needed and read with l2 only); the other arguments as there.
    Returns dx [B, L, H * d] (`out` may be a slice of a fused gradient)."""
    dt, dev = _storage(dout, "dout")
    if layout == "heads":
        if H < 1 or dout.dim() != 3 or dout.shape[0] % H:
            raise ValueError("dout must be [B * H, L, d], H at least 1")
        B, L, d = dout.shape[0] // H, dout.shape[1], dout.shape[2]
    else:
        if H < 1 or dout.dim() != 3 or dout.shape[2] % H:
            raise ValueError("dout must be [B, L, H * d], H at least 1")
        B, L, d = dout.shape[0], dout.shape[1], dout.shape[2] // H
    _require(dout, "dout", dt, dev)
    o = _rope_args(inv_freq, axes, H, B, L, d, positions, grid, frame_offset, interleaved, l2,
                   layout, dev)
    if l2 and x is None:
        raise ValueError("x is needed with l2")
    if not l2:
        x = None  # not read
    for t, n in ((x, "x"), (out, "out")):
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or t.dtype is not dt or t.device != dev or \
                tuple(t.shape) != (B, L, H * d):
            raise ValueError(f"{n} must be {dt} [{B}, {L}, {H * d}] on {dev}")
        row = _token_rows(t, n, H)
        if n == "x":
            o.x_row_stride = row
        else:
            o.dx_row_stride = row
    if out is None:
        out = _new((B, L, H * d), dt, dev, stream)
    st = _call(lib.vda_rope_backward, dev, dout.data_ptr(), _ptr(x), inv_freq.data_ptr(),
               _ptr(positions), B, L, H, d, ctypes.byref(o), int(dt == torch.float32),
               out.data_ptr(), _stream_ptr(dev, stream))
    _check(st, "vda_rope_backward")
    return out
