"""Python binding of libstreamkl.so (the C ABI declared in include/streamkl.h).

Argument marshalling only: every step of the forward and backward pass runs
in the library's gfx950 kernels. PyTorch provides device memory and the
current HIP stream. Importing this module fails loudly when the library has
not been built; there is no fallback implementation.

    kl, lse1, lse2 = fwd(q1, k1, q2, k2, s1, s2, causal, direction)
    kl, lse1, lse2 = fwd_split(q1, k1, q2, k2, s1, s2, causal, direction, splits="auto")
    dQ1, dK1, dQ2, dK2 = bwd(q1, k1, q2, k2, kl, lse1, lse2, dkl, ..., want=("dq2", "dk2"), strategy="auto")
    loss = attention_kl(q1, k1, q2, k2, causal=True).mean(); loss.backward()

The operators around it:

    yq, yk = qk_norm_rope(q, k, wq, wk, rope_table(n, rot))           # projections -> normed, rotated, head-major
    loss = attention_kl_proj(q1, k1, q2, k2, QKPrep(...), QKPrep(...), causal=True).mean()
    out = diff_attention(q1, k1, q2, k2, v, lam, causal=True)         # (softmax map 1 - lam * softmax map 2) v

The operators on rows of logits:

    scores = token_logprobs(logits, tokens, top=20)                   # logp, entropy, lse, top_logp, top_ids
    best = token_logprobs(teacher_logits, top=64)
    loss = topk_distill_loss(student_logits, best.top_ids, best.top_logp)
"""
from __future__ import annotations

import ctypes
import math
import os
import typing

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libstreamkl.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_HIP, ERR_SCRATCH_LIMIT = 0, 1, 2, 3, 4
NOALLOC_SCRATCH_BYTES = 16 << 20
FWD, REV = 0, 1
BWD_AUTO, BWD_SEPARATE, BWD_FUSED = 0, 1, 2
GRAD_BITS = {"dq1": 1, "dk1": 2, "dq2": 4, "dk2": 8}
ACT_SOFTMAX, ACT_SIGMOID = 0, 1
ENTRY_POINTS = ("streamkl_fwd", "streamkl_bwd", "streamkl_bwd_ex", "streamkl_bwd_choose", "streamkl_fwd_split",
                "streamkl_fwd_split_noalloc", "streamkl_fwd_split_workspace_bytes", "streamkl_fwd_split_count",
                "streamkl_fwd_act", "streamkl_bwd_act", "streamkl_bwd_grads", "streamkl_strerror", "streamkl_version",
                "streamkl_supported_head_dim", "streamkl_qk_norm_rope_fwd", "streamkl_qk_norm_rope_bwd",
                "streamkl_qk_norm_rope_bwd_workspace_bytes", "streamkl_diff_fwd", "streamkl_diff_fwd_split_count",
                "streamkl_diff_fwd_workspace_bytes", "streamkl_diff_bwd", "streamkl_diff_bwd_workspace_bytes",
                "streamkl_token_logprobs_fwd", "streamkl_token_logprobs_workspace_bytes", "streamkl_token_logprobs_bwd",
                "streamkl_topk_distill_fwd", "streamkl_topk_distill_workspace_bytes", "streamkl_topk_distill_bwd",
                "streamkl_topk_distill_step", "streamkl_topk_distill_total")
_MAX_INT = 0x7fffffff   # the ABI's extents; ctypes would cut a larger one silently
DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class _Rows(ctypes.Structure):
    """streamkl_rows: a [batch, head, row] arrangement of contiguous rows."""
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_longlong), ("sh", ctypes.c_longlong),
                ("sn", ctypes.c_longlong)]


class _Logits(ctypes.Structure):
    """streamkl_logits: B N rows of V logits."""
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_longlong), ("sn", ctypes.c_longlong), ("B", ctypes.c_int),
                ("N", ctypes.c_int), ("V", ctypes.c_int), ("dtype", ctypes.c_int)]


class _TeacherList(ctypes.Structure):
    """streamkl_teacher_list: a teacher's best tokens."""
    _fields_ = [("ids", ctypes.c_void_p), ("values", ctypes.c_void_p), ("K", ctypes.c_int), ("ids64", ctypes.c_int),
                ("dtype", ctypes.c_int), ("rest", ctypes.c_int), ("scale", ctypes.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_20005_amd.build` "
                          "(the attention-KL primitive has no non-HIP implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.streamkl_fwd.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, vp, vp, vp, vp]
    lib.streamkl_fwd.restype = i
    lib.streamkl_bwd.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.streamkl_bwd.restype = i
    lib.streamkl_bwd_ex.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, vp, vp, vp, vp, vp, vp, vp, vp, i,
                                    vp]
    lib.streamkl_bwd_ex.restype = i
    lib.streamkl_fwd_act.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, i, vp, vp, vp, vp]
    lib.streamkl_fwd_act.restype = i
    lib.streamkl_bwd_act.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, i, vp, vp, vp, vp, vp, vp, vp,
                                     vp, vp]
    lib.streamkl_bwd_act.restype = i
    lib.streamkl_bwd_grads.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, i, vp, vp, vp, vp, vp, vp, vp,
                                       vp, i, i, vp]
    lib.streamkl_bwd_grads.restype = i
    lib.streamkl_bwd_choose.argtypes = [i, i, i, i, i, i, i, i, i]
    lib.streamkl_bwd_choose.restype = i
    sz = ctypes.c_size_t
    lib.streamkl_fwd_split.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, i, vp, sz, vp, vp, vp, vp]
    lib.streamkl_fwd_split.restype = i
    lib.streamkl_fwd_split_noalloc.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, f, i, i, i, vp, vp, vp, vp]
    lib.streamkl_fwd_split_noalloc.restype = i
    lib.streamkl_fwd_split_workspace_bytes.argtypes = [i, i, i, i]
    lib.streamkl_fwd_split_workspace_bytes.restype = sz
    lib.streamkl_fwd_split_count.argtypes = [i, i, i, i, i, i]
    lib.streamkl_fwd_split_count.restype = i
    rows = ctypes.POINTER(_Rows)
    lib.streamkl_qk_norm_rope_fwd.argtypes = [rows, rows, i, i, i, i, i, i, i, vp, vp, f, vp, i, i, i, vp, vp, i, i, i,
                                              i, vp, vp, vp]
    lib.streamkl_qk_norm_rope_fwd.restype = i
    lib.streamkl_qk_norm_rope_bwd.argtypes = [rows, rows, i, i, i, i, i, i, i, vp, vp, f, vp, i, i, i, vp, vp, i, i, i,
                                              i, vp, vp, i, vp, sz, vp, vp, vp, vp, vp]
    lib.streamkl_qk_norm_rope_bwd.restype = i
    lib.streamkl_qk_norm_rope_bwd_workspace_bytes.argtypes = [i, i, i, i, i, i]
    lib.streamkl_qk_norm_rope_bwd_workspace_bytes.restype = sz
    lib.streamkl_diff_fwd.argtypes = [rows, rows, rows, rows, rows, i, i, i, i, i, i, i, f, i, vp, vp, vp, i, vp, sz,
                                      vp, vp, vp, vp, vp]
    lib.streamkl_diff_fwd.restype = i
    lib.streamkl_diff_fwd_split_count.argtypes = [i, i, i, i, i, i, i, i]
    lib.streamkl_diff_fwd_split_count.restype = i
    lib.streamkl_diff_fwd_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.streamkl_diff_fwd_workspace_bytes.restype = sz
    lib.streamkl_diff_bwd.argtypes = [rows, rows, rows, rows, rows, i, i, i, i, i, i, i, f, i, vp, vp, vp, vp, vp, vp,
                                      vp, vp, vp, sz, vp, vp, vp, vp, vp, vp, i, vp]
    lib.streamkl_diff_bwd.restype = i
    lib.streamkl_diff_bwd_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    lib.streamkl_diff_bwd_workspace_bytes.restype = sz
    logits, teacher, ll = ctypes.POINTER(_Logits), ctypes.POINTER(_TeacherList), ctypes.c_longlong
    lib.streamkl_token_logprobs_fwd.argtypes = [logits, vp, i, f, i, vp, sz, vp, vp, vp, vp, vp, vp, vp]
    lib.streamkl_token_logprobs_fwd.restype = i
    lib.streamkl_token_logprobs_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.streamkl_token_logprobs_workspace_bytes.restype = sz
    lib.streamkl_token_logprobs_bwd.argtypes = [logits, vp, i, f, vp, vp, vp, vp, vp, vp, vp, ll, ll, vp]
    lib.streamkl_token_logprobs_bwd.restype = i
    lib.streamkl_topk_distill_fwd.argtypes = [logits, teacher, f, i, vp, sz, vp, vp, vp]
    lib.streamkl_topk_distill_fwd.restype = i
    lib.streamkl_topk_distill_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.streamkl_topk_distill_workspace_bytes.restype = sz
    lib.streamkl_topk_distill_bwd.argtypes = [logits, teacher, f, i, vp, vp, f, vp, i, vp, ll, ll, vp]
    lib.streamkl_topk_distill_bwd.restype = i
    lib.streamkl_topk_distill_step.argtypes = [logits, teacher, f, i, vp, sz, vp, f, vp, vp, vp, ll, ll, vp]
    lib.streamkl_topk_distill_step.restype = i
    lib.streamkl_topk_distill_total.argtypes = [vp, vp, f, ll, vp, vp]
    lib.streamkl_topk_distill_total.restype = i
    lib.streamkl_strerror.argtypes = [i]
    lib.streamkl_strerror.restype = ctypes.c_char_p
    lib.streamkl_version.argtypes = []
    lib.streamkl_version.restype = ctypes.c_char_p
    lib.streamkl_supported_head_dim.argtypes = [i]
    lib.streamkl_supported_head_dim.restype = i
    return lib


lib = _load()


class StreamKLError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib.streamkl_strerror(status).decode()} (status {status})")


def version() -> str:
    return lib.streamkl_version().decode()


def supported_head_dim(d: int) -> bool:
    return bool(lib.streamkl_supported_head_dim(int(d)))


def _p(t):
    return None if t is None else t.data_ptr()   # converted by argtypes


def _stream(dev):
    """The raw current stream of dev, without the Stream object that torch.cuda.current_stream builds (2 us a call)."""
    return torch._C._cuda_getCurrentRawStream(dev.index)


class _SameDevice:
    """Stands in for torch.cuda.device(dev) where dev is current already (1.5 us a call)."""

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return False


_SAME_DEVICE = _SameDevice()


def _on(dev):
    """Context in which dev is the current device."""
    return _SAME_DEVICE if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def _rows3(out, shape, dev, names):
    """The three row outputs: new ones, or the caller's after a check."""
    if out is None:
        return (torch.empty(shape, dtype=torch.float32, device=dev), torch.empty(shape, dtype=torch.float32, device=dev),
                torch.empty(shape, dtype=torch.float32, device=dev))
    return tuple(_f32_rows(t, shape, dev, n) for t, n in zip(out, names))


def _direction(direction) -> int:
    if direction in (FWD, "fwd", "forward"):
        return FWD
    if direction in (REV, "rev", "reverse"):
        return REV
    raise ValueError(f"direction must be 'fwd' (KL(P1||P2)) or 'rev' (KL(P2||P1)), got {direction!r}")


def _check_inputs(q1, k1, q2, k2):
    for n, t in (("q1", q1), ("k1", k1), ("q2", q2), ("k2", k2)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError(f"{n} must be a GPU tensor")
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{n} must be bfloat16, got {t.dtype}")
        if t.dim() != 4 or not t.is_contiguous():
            raise ValueError(f"{n} must be a contiguous [B, H, N, d] tensor")
    B, H, NQ, d1 = q1.shape
    NK = k1.shape[2]
    d2 = q2.shape[3]
    if tuple(k1.shape) != (B, H, NK, d1) or tuple(q2.shape) != (B, H, NQ, d2) or tuple(k2.shape) != (B, H, NK, d2):
        raise ValueError(f"inconsistent shapes q1{tuple(q1.shape)} k1{tuple(k1.shape)} "
                         f"q2{tuple(q2.shape)} k2{tuple(k2.shape)}")
    if len({q1.device, k1.device, q2.device, k2.device}) != 1:
        raise ValueError("all inputs must be on one device")
    return B, H, NQ, NK, d1, d2


def _scales(s1, s2, d1, d2):
    return (1.0 / math.sqrt(d1) if s1 is None else float(s1)), (1.0 / math.sqrt(d2) if s2 is None else float(s2))


def _f32_rows(t, shape, dev, name):
    if t is None:
        return None
    if t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape {shape} on {dev}")
    return t


def fwd(q1, k1, q2, k2, s1=None, s2=None, causal=False, direction=FWD, out=None):
    """streamkl_fwd: returns (kl, lse1, lse2), float32 [B, H, N_Q].

    s_t defaults to 1/sqrt(d_t). ``out`` may hold three preallocated tensors.
    """
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    s1, s2 = _scales(s1, s2, d1, d2)
    dev = q1.device
    kl, lse1, lse2 = _rows3(out, (B, H, NQ), dev, ("kl", "lse1", "lse2"))
    with _on(dev):
        st = lib.streamkl_fwd(_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2,
                              int(bool(causal)), _direction(direction), _p(kl), _p(lse1), _p(lse2), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_fwd")
    return kl, lse1, lse2


def _activation(activation) -> int:
    if activation in (ACT_SOFTMAX, "softmax"):
        return ACT_SOFTMAX
    if activation in (ACT_SIGMOID, "sigmoid"):
        return ACT_SIGMOID
    raise ValueError(f"activation must be 'softmax' or 'sigmoid', got {activation!r}")


def fwd_act(q1, k1, q2, k2, s1=None, s2=None, causal=False, direction=FWD, activation="sigmoid", out=None):
    """streamkl_fwd_act: returns (kl, stat1, stat2), float32 [B, H, N_Q].

    activation "softmax": exactly fwd (the stats are the LSEs). "sigmoid":
    unnormalised sigmoid scores, kl is the generalized KL of the two score
    rows and the stats are the row masses sum_j sigmoid(S_t[j]).
    """
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    s1, s2 = _scales(s1, s2, d1, d2)
    dev = q1.device
    kl, st1, st2 = _rows3(out, (B, H, NQ), dev, ("kl", "stat1", "stat2"))
    with _on(dev):
        st = lib.streamkl_fwd_act(_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2, int(bool(causal)),
                                  _direction(direction), _activation(activation), _p(kl), _p(st1), _p(st2),
                                  _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_fwd_act")
    return kl, st1, st2


def split_count(B, H, n_q, n_k, d1, d2) -> int:
    """streamkl_fwd_split_count: the adaptive split count of Sec. 3.3 (0 for invalid arguments)."""
    return int(lib.streamkl_fwd_split_count(int(B), int(H), int(n_q), int(n_k), int(d1), int(d2)))


def split_workspace_bytes(B, H, n_q, splits) -> int:
    """streamkl_fwd_split_workspace_bytes: workspace the split-K forward needs."""
    return int(lib.streamkl_fwd_split_workspace_bytes(int(B), int(H), int(n_q), int(splits)))


def fwd_split(q1, k1, q2, k2, s1=None, s2=None, causal=False, direction=FWD, splits="auto", out=None,
              workspace=None):
    """streamkl_fwd_split: the split-K forward; returns (kl, lse1, lse2) like fwd.

    splits: an int >= 1 or "auto" (split_count). The workspace is allocated
    here unless ``workspace`` (a device tensor of at least split_workspace_bytes
    bytes) is given.
    """
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    s1, s2 = _scales(s1, s2, d1, d2)
    dev = q1.device
    w = split_count(B, H, NQ, NK, d1, d2) if splits == "auto" else int(splits)
    kl, lse1, lse2 = _rows3(out, (B, H, NQ), dev, ("kl", "lse1", "lse2"))
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
    elif w == 1:   # the single pass needs none
        ws_bytes = 0
    else:
        ws_bytes = max(split_workspace_bytes(B, H, NQ, w), 4)
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        st = lib.streamkl_fwd_split(_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2,
                                    int(bool(causal)), _direction(direction), w, _p(workspace), ws_bytes,
                                    _p(kl), _p(lse1), _p(lse2), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_fwd_split")
    return kl, lse1, lse2


def fwd_split_noalloc(q1, k1, q2, k2, s1=None, s2=None, causal=False, direction=FWD, splits="auto", out=None):
    """streamkl_fwd_split_noalloc: the split-K forward with its partial row
    statistics in the library's static per-GPU scratch (nothing is allocated
    for them); returns (kl, lse1, lse2) like fwd_split. Outputs are allocated
    here unless ``out`` is given."""
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    s1, s2 = _scales(s1, s2, d1, d2)
    dev = q1.device
    w = split_count(B, H, NQ, NK, d1, d2) if splits == "auto" else int(splits)
    kl, lse1, lse2 = _rows3(out, (B, H, NQ), dev, ("kl", "lse1", "lse2"))
    with _on(dev):
        st = lib.streamkl_fwd_split_noalloc(_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2,
                                            int(bool(causal)), _direction(direction), w, _p(kl), _p(lse1),
                                            _p(lse2), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_fwd_split_noalloc")
    return kl, lse1, lse2


_STRATEGIES = {"auto": BWD_AUTO, "separate": BWD_SEPARATE, "fused": BWD_FUSED}


def _strategy(strategy) -> int:
    if isinstance(strategy, str):
        if strategy not in _STRATEGIES:
            raise ValueError(f"strategy must be one of {sorted(_STRATEGIES)}, got {strategy!r}")
        return _STRATEGIES[strategy]
    return int(strategy)


def bwd_choose(B, H, n_q, n_k, d1, d2, causal=False, direction=FWD, want=("dq2", "dk2")) -> str:
    """streamkl_bwd_choose: the strategy ("separate" or "fused") the adaptive rule picks."""
    bits = 0
    for n in want:
        bits |= GRAD_BITS[n]
    r = lib.streamkl_bwd_choose(B, H, n_q, n_k, d1, d2, int(bool(causal)), _direction(direction), bits)
    if r == 0:
        raise StreamKLError(ERR_INVALID_ARG, "streamkl_bwd_choose")
    return "fused" if r == BWD_FUSED else "separate"


def bwd(q1, k1, q2, k2, kl, lse1, lse2, dkl=None, s1=None, s2=None, causal=False, direction=FWD,
        want=("dq2", "dk2"), out=None, strategy="separate", activation="softmax"):
    """streamkl_bwd / streamkl_bwd_ex / streamkl_bwd_act: returns (dQ1, dK1, dQ2, dK2), float32, None where not
    requested.

    want: any of "dq1", "dk1", "dq2", "dk2". dkl: per-row upstream gradient
    (float32 [B, H, N_Q]) or None for all ones. ``out`` may map those names to
    preallocated tensors. strategy: "separate" (streamkl_bwd, reproducible),
    "fused" (one kernel, dQ by atomics) or "auto" (the adaptive rule).
    activation "sigmoid" (streamkl_bwd_act, separate kernels): kl, lse1, lse2
    are not needed and may be None.
    """
    act = _activation(activation)
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    s1, s2 = _scales(s1, s2, d1, d2)
    dev = q1.device
    rows = (B, H, NQ)
    kl, lse1, lse2 = (_f32_rows(t, rows, dev, n) for t, n in ((kl, "kl"), (lse1, "lse1"), (lse2, "lse2")))
    dkl = _f32_rows(dkl, rows, dev, "dkl")
    shapes = {"dq1": (B, H, NQ, d1), "dk1": (B, H, NK, d1), "dq2": (B, H, NQ, d2), "dk2": (B, H, NK, d2)}
    unknown = set(want) - set(shapes)
    if unknown:
        raise ValueError(f"unknown gradient names {sorted(unknown)}")
    out = dict(out or {})
    grads = {}
    for n in ("dq1", "dk1", "dq2", "dk2"):
        if n in want:
            t = out.get(n)
            grads[n] = _f32_rows(t, shapes[n], dev, n) if t is not None else \
                torch.empty(shapes[n], dtype=torch.float32, device=dev)
        else:
            grads[n] = None
    strat = _strategy(strategy)
    args = (_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2, int(bool(causal)), _direction(direction),
            _p(kl), _p(lse1), _p(lse2), _p(dkl), _p(grads["dq1"]), _p(grads["dk1"]), _p(grads["dq2"]),
            _p(grads["dk2"]))
    with _on(dev):
        if act == ACT_SIGMOID:
            if strat != BWD_SEPARATE:
                raise ValueError("sigmoid scores run the separate backward kernels only")
            st, where = lib.streamkl_bwd_act(*args[:14], act, *args[14:], _stream(dev)), "streamkl_bwd_act"
        elif strat == BWD_SEPARATE:
            st, where = lib.streamkl_bwd(*args, _stream(dev)), "streamkl_bwd"
        else:
            st, where = lib.streamkl_bwd_ex(*args, strat, _stream(dev)), "streamkl_bwd_ex"
    if st != OK:
        raise StreamKLError(st, where)
    return grads["dq1"], grads["dk1"], grads["dq2"], grads["dk2"]


def _bwd_bf16(q1, k1, q2, k2, kl, stat1, stat2, g, s1, s2, causal, direction, names, strat, act):
    """streamkl_bwd_grads: the gradients named in ``names`` in the inputs' bf16, written so by the kernels (a float32
    gradient and its cast would pass over memory three times more). The fused strategy adds into a float32 dQ, the
    small side where it applies, which is cast here. The tensors are checked again: a saved-tensor hook may have put
    others in their place since the forward pass."""
    B, H, NQ, NK, d1, d2 = _check_inputs(q1, k1, q2, k2)
    kl, stat1, stat2, g = (_f32_rows(t, (B, H, NQ), q1.device, n)
                           for t, n in ((kl, "kl"), (stat1, "lse1"), (stat2, "lse2"), (g, "dkl")))
    if strat == BWD_AUTO:
        strat = BWD_FUSED if bwd_choose(B, H, NQ, NK, d1, d2, causal, direction, names) == "fused" else BWD_SEPARATE
    dev = q1.device
    shapes = {"dq1": q1.shape, "dk1": k1.shape, "dq2": q2.shape, "dk2": k2.shape}
    grads, bits = dict.fromkeys(shapes), 0
    for n in names:
        half = strat != BWD_FUSED or n in ("dk1", "dk2")
        grads[n] = torch.empty(shapes[n], dtype=torch.bfloat16 if half else torch.float32, device=dev)
        bits |= GRAD_BITS[n] if half else 0
    with _on(dev):
        st = lib.streamkl_bwd_grads(_p(q1), _p(k1), _p(q2), _p(k2), B, H, NQ, NK, d1, d2, s1, s2, int(bool(causal)),
                                    _direction(direction), act, _p(kl), _p(stat1), _p(stat2), _p(g),
                                    _p(grads["dq1"]), _p(grads["dk1"]), _p(grads["dq2"]), _p(grads["dk2"]), bits,
                                    strat, _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_bwd_grads")
    return tuple(t if t is None else t.to(torch.bfloat16) for t in grads.values())


class _AttentionKL(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q1, k1, q2, k2, s1, s2, causal, direction, bwd_strategy, act):
        if act == ACT_SIGMOID:
            kl, st1, st2 = fwd_act(q1, k1, q2, k2, s1, s2, causal, direction, ACT_SIGMOID)
        else:
            # the adaptive split count is 1 (the single-pass kernel) unless the heads have few query rows
            kl, st1, st2 = fwd_split(q1, k1, q2, k2, s1, s2, causal, direction, splits="auto")
        ctx.save_for_backward(q1, k1, q2, k2, kl, st1, st2)
        ctx.cfg = (s1, s2, causal, direction, bwd_strategy, act)
        ctx.mark_non_differentiable(st1, st2)
        return kl, st1, st2

    @staticmethod
    def backward(ctx, gkl, _g1, _g2):
        q1, k1, q2, k2, kl, st1, st2 = ctx.saved_tensors
        s1, s2, causal, direction, strategy, act = ctx.cfg
        names = [n for n, need in zip(("dq1", "dk1", "dq2", "dk2"), ctx.needs_input_grad[:4]) if need]
        if not names:
            return (None,) * 10
        g = gkl.to(torch.float32).contiguous()
        return (*_bwd_bf16(q1, k1, q2, k2, kl, st1, st2, g, s1, s2, causal, direction, names,
                           BWD_SEPARATE if act == ACT_SIGMOID else _strategy(strategy), act),
                None, None, None, None, None, None)


def attention_kl(q1, k1, q2, k2, *, s1=None, s2=None, causal=False, direction="fwd", return_lse=False,
                 bwd_strategy="auto", activation="softmax"):
    """Per-row KL between softmax(s1 q1 k1^T) and softmax(s2 q2 k2^T), differentiable.

    Returns kl [B, H, N_Q] (and the two row statistics if ``return_lse``:
    lse1, lse2 for softmax, the row masses for sigmoid). The paper's training
    objective is ``attention_kl(...).mean()``. Gradients flow to the inputs
    that require them: (q2, k2) in standard distillation (Setting 1),
    (q1, k1) when the first distribution is trained (Setting 2), or both.
    bwd_strategy: "auto" (the adaptive rule of streamkl_bwd_choose), "fused"
    or "separate" (bitwise reproducible gradients). activation "sigmoid":
    unnormalised sigmoid scores and the generalized KL (streamkl_fwd_act).
    """
    d1, d2 = q1.shape[-1], q2.shape[-1]
    s1, s2 = _scales(s1, s2, d1, d2)
    _strategy(bwd_strategy)
    kl, st1, st2 = _AttentionKL.apply(q1, k1, q2, k2, s1, s2, bool(causal), _direction(direction), bwd_strategy,
                                      _activation(activation))
    return (kl, st1, st2) if return_lse else kl


def _differentiated(*tensors):
    """Whether autograd has to see a call: an input requires a gradient, or may carry a tangent of forward mode (for which
    the autograd functions have no formula, and raise)."""
    if forward_ad._current_level >= 0:   # inside dual_level()
        return True
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _upstream(g):
    """An upstream gradient as the kernels read it: contiguous, 16-byte aligned (a part of a concatenation's need not be)."""
    g = g.contiguous()
    return g.clone() if g.data_ptr() & 15 else g


# --- norms of queries and keys with the position rotation -------------------------------------------------------------


def rope_table(n_pos, rot_dim, base=10000.0, device="cuda"):
    """Cosines and sines of the positions 0 .. n_pos - 1 for qk_norm_rope: float32 [n_pos, rot_dim], the rot_dim/2
    cosines of a position, then its sines. Pair i turns by p * base^(-2 i / rot_dim). The angles are formed in
    64 bits (at position 100000 a float32 angle is off by up to 4e-3) and the values rounded once. A program lays this
    out once."""
    if rot_dim <= 0 or rot_dim % 16 != 0:
        raise ValueError(f"rot_dim must be a positive multiple of 16, got {rot_dim}")
    pos = torch.arange(int(n_pos), device=device, dtype=torch.float64)
    freq = float(base) ** (torch.arange(0, rot_dim, 2, device=device, dtype=torch.float64) / -rot_dim)
    angle = pos[:, None] * freq[None, :]
    return torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()


def _rows(t, name, batch=0, head=1, row=2):
    """A tensor with contiguous 16-byte aligned rows as a streamkl_rows; batch, head and row are its axes."""
    n, st, p = t.shape, t.stride(), t.data_ptr()
    if st[3] != 1 and n[3] != 1:
        raise ValueError(f"{name} must be contiguous along its last axis")
    # the stride of an extent of one says nothing
    sb, sh, sn = st[batch] if n[batch] > 1 else 0, st[head] if n[head] > 1 else 0, st[row] if n[row] > 1 else 0
    if p & 15 or (sb | sh | sn) & (3 if t.dtype is torch.float32 else 7):
        raise ValueError(f"the rows of {name} must begin at multiples of 16 bytes")
    return _Rows(p, sb, sh, sn)


def _bf16_out(t, shape, dev, name):
    if t is None:
        return torch.empty(shape, dtype=torch.bfloat16, device=dev)
    if t.dtype is not torch.bfloat16 or t.shape != shape or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous bfloat16 tensor of shape {shape} on {dev}")
    return t


def _workspace(t, dev):
    """A caller's workspace, checked: its bytes."""
    if not (isinstance(t, torch.Tensor) and t.device == dev and t.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    return t.numel() * t.element_size()


def _prep_error(q, k):
    """What is wrong with the tensors of a norm-and-rotation call."""
    for n, t in (("q", q), ("k", k)):
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            return ValueError(f"{n} must be a GPU tensor")
        if t.dtype not in DTYPES:
            return ValueError(f"{n} must be bfloat16, float16 or float32, got {t.dtype}")
        if t.dim() != 4:
            return ValueError(f"{n} must be a [B, N, H, d] tensor")
    return ValueError("q and k must have one type, device, batch and head dim")


def _prep_inputs(q, k, wq, wk, table, q_positions, k_positions, expand_k):
    """Checked arguments of the norm-and-rotation calls: (device, B, H, HK, N_Q, N_K, d, n_pos, rot, copies)."""
    first = k if q is None else q
    if first is None:
        raise ValueError("q and k are both None")
    if not (isinstance(first, torch.Tensor) and first.is_cuda and first.dim() == 4 and first.dtype in DTYPES):
        raise _prep_error(q, k)
    dev = first.device
    B, N, heads, d = first.shape
    NQ, H, NK, HK = (0, 0, N, heads) if q is None else (N, heads, 0, 0)
    if q is not None and k is not None:
        if not (isinstance(k, torch.Tensor) and k.dtype is first.dtype and k.device == dev and k.dim() == 4):
            raise _prep_error(q, k)
        kb, NK, HK, kd = k.shape
        if kb != B or kd != d:
            raise _prep_error(q, k)
    for n, w in (("wq", wq), ("wk", wk)):
        if w is not None and not (w.dtype is torch.float32 and w.shape == (d,) and w.is_contiguous() and
                                  w.device == dev):
            raise ValueError(f"{n} must be a contiguous float32 tensor of shape {(d,)} on {dev}")
    n_pos = rot = 0
    if table is not None:
        if not (table.dtype is torch.float32 and table.dim() == 2 and table.is_contiguous() and table.device == dev):
            raise ValueError(f"table must be a contiguous float32 [positions, rot_dim] tensor on {dev}")
        n_pos, rot = table.shape
        if rot <= 0 or rot > d or rot % 16:
            raise ValueError(f"the table's rot_dim must be a multiple of 16 up to the head dim {d}, got {rot}")
    for n, p, t, rows in (("q_positions", q_positions, q, NQ), ("k_positions", k_positions, k, NK)):
        if p is None:
            continue
        if t is None:
            raise ValueError(f"{n} given without {n[0]}")
        if p.dtype not in (torch.int32, torch.int64) or (p.shape != (B, rows) and p.shape != (rows,)) or \
                not p.is_contiguous() or p.device != dev:
            raise ValueError(f"{n} must be a contiguous int32 or int64 tensor of shape {(rows,)} or {(B, rows)} on "
                             f"{dev}")
    if q_positions is not None and k_positions is not None and q_positions.dtype != k_positions.dtype:
        raise ValueError("q_positions and k_positions must have one type")
    if B > _MAX_INT or NQ > _MAX_INT or NK > _MAX_INT or H > _MAX_INT or HK > _MAX_INT or n_pos > _MAX_INT:
        raise ValueError("an extent does not fit 31 bits")
    if NQ > NK and table is not None and k is not None and q is not None and q_positions is None:
        raise ValueError("more queries than keys: their positions have to be given")
    if (NQ > n_pos or NK > n_pos) and table is not None:   # the last places of rows without positions
        for n, p, t, last in (("q", q_positions, q, NQ if k is None else NK), ("k", k_positions, k, NK)):
            if p is None and t is not None and t.numel() and last > n_pos:
                raise ValueError(f"{n} reaches position {last - 1}, the table holds {n_pos}")
    copies = 1
    if expand_k:
        if q is None or k is None or HK == 0 or H % HK:
            raise ValueError("expand_k needs q and k, with whole groups of query heads per key head")
        copies = H // HK
    return dev, B, H, HK, NQ, NK, d, n_pos, rot, copies


def _prep_args(q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, cfg):
    """The arguments that the forward and backward calls share."""
    _, B, H, HK, NQ, NK, d, n_pos, rot, copies = cfg
    pos = q_positions if q_positions is not None else k_positions
    return (None if q is None else _rows(q, "q", 0, 2, 1), None if k is None else _rows(k, "k", 0, 2, 1), B, H, HK, NQ,
            NK, d, DTYPES[(q if q is not None else k).dtype], _p(wq), _p(wk), float(eps), _p(table), n_pos, rot,
            int(bool(interleaved)), _p(q_positions), _p(k_positions),
            int(pos is not None and pos.dtype == torch.int64), int(q_positions is not None and q_positions.dim() == 1),
            int(k_positions is not None and k_positions.dim() == 1), copies)


def qk_norm_rope_fwd(q, k, wq=None, wk=None, table=None, eps=1e-6, q_positions=None, k_positions=None,
                     interleaved=False, expand_k=False, out=None):
    """streamkl_qk_norm_rope_fwd: (yq, yk), bf16 [B, H, N, d]; None for a side that is None. See qk_norm_rope.
    ``out`` may hold the two outputs, preallocated."""
    cfg = _prep_inputs(q, k, wq, wk, table, q_positions, k_positions, expand_k)
    dev, B, H, HK, NQ, NK, d, _, _, copies = cfg
    yq, yk = out or (None, None)
    yq = None if q is None else _bf16_out(yq, (B, H, NQ, d), dev, "yq")
    yk = None if k is None else _bf16_out(yk, (B, HK * copies, NK, d), dev, "yk")
    args = _prep_args(q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, cfg)
    with _on(dev):
        st = lib.streamkl_qk_norm_rope_fwd(*args, _p(yq), _p(yk), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_qk_norm_rope_fwd")
    return yq, yk


def qk_norm_rope_bwd(q, k, dyq, dyk, wq=None, wk=None, table=None, eps=1e-6, q_positions=None, k_positions=None,
                     interleaved=False, expand_k=False, want_w=True, workspace=None):
    """streamkl_qk_norm_rope_bwd: (dq, dk, dwq, dwk) from the upstream gradients dyq, dyk (contiguous, both bf16 or both
    float32, in the layout of the outputs); dq and dk in the inputs' type, dwq and dwk float32 (None unless
    ``want_w``). The workspace is allocated here unless given."""
    cfg = _prep_inputs(q, k, wq, wk, table, q_positions, k_positions, expand_k)
    dev, B, H, HK, NQ, NK, d, _, _, copies = cfg
    shapes = (None if q is None else (B, H, NQ, d), None if k is None else (B, HK * copies, NK, d))
    kind = getattr(dyq if q is not None else dyk, "dtype", None)
    for n, shape, t in zip(("dyq", "dyk"), shapes, (dyq, dyk)):
        if (shape is None) != (t is None):
            raise ValueError(f"{n} must be given exactly where {n[-1]} is")
        if t is not None and (t.dtype not in (torch.bfloat16, torch.float32) or t.dtype != kind or
                              tuple(t.shape) != shape or not t.is_contiguous() or t.device != dev):
            raise ValueError(f"{n} must be a contiguous bfloat16 or float32 tensor of shape {shape} on {dev}, of one "
                             "type with the other")
    dx = [None if t is None else torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k)]
    dw = [None if t is None or not want_w else torch.empty(d, dtype=torch.float32, device=dev) for t in (q, k)]
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = _workspace(workspace, dev)
    elif want_w:
        ws_bytes = lib.streamkl_qk_norm_rope_bwd_workspace_bytes(B, H, HK, NQ, NK, d)
        workspace = torch.empty(max(ws_bytes, 4), dtype=torch.uint8, device=dev)
    args = _prep_args(q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, cfg)
    with _on(dev):
        st = lib.streamkl_qk_norm_rope_bwd(*args, _p(dyq), _p(dyk), DTYPES[kind], _p(workspace), ws_bytes, _p(dx[0]),
                                           _p(dx[1]), _p(dw[0]), _p(dw[1]), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_qk_norm_rope_bwd")
    return dx[0], dx[1], dw[0], dw[1]


class _QKNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, expand_k):
        ctx.save_for_backward(q, k, wq, wk, table, q_positions, k_positions)
        ctx.cfg = (eps, interleaved, expand_k)
        ctx.set_materialize_grads(False)
        return qk_norm_rope_fwd(q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, expand_k)

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        q, k, wq, wk, table, q_positions, k_positions = ctx.saved_tensors
        eps, interleaved, expand_k = ctx.cfg
        need = ctx.needs_input_grad
        if gq is None and gk is None:
            return (None,) * 10
        # the gradient of an output that the loss does not reach is zero
        if gq is None and q is not None:
            gq = torch.zeros((q.shape[0], q.shape[2], q.shape[1], q.shape[3]), dtype=torch.bfloat16, device=q.device)
        if gk is None and k is not None:
            heads = q.shape[2] if expand_k else k.shape[2]
            gk = torch.zeros((k.shape[0], heads, k.shape[1], k.shape[3]), dtype=torch.bfloat16, device=k.device)
        gq, gk = (None if g is None else _upstream(g) for g in (gq, gk))
        dq, dk, dwq, dwk = qk_norm_rope_bwd(q, k, gq, gk, wq, wk, table, eps, q_positions, k_positions, interleaved,
                                            expand_k, want_w=need[2] or need[3])
        return (dq if need[0] else None, dk if need[1] else None, dwq if need[2] else None, dwk if need[3] else None,
                *(None,) * 6)


def qk_norm_rope(q, k, wq=None, wk=None, table=None, *, eps=1e-6, q_positions=None, k_positions=None,
                 interleaved=False, expand_k=False):
    """Norm of every query and key head and the rotation by its position, differentiable; one kernel.

    q [B, N_Q, H, d] and k [B, N_K, HK, d] as their projections leave them (bfloat16, float16 or float32; any strides
    with a contiguous last axis), either may be None. Returns yq [B, H, N_Q, d] and yk [B, HK, N_K, d] in bf16,
    contiguous, as attention_kl and diff_attention read them:
        n = x / sqrt(mean(x^2) + eps) * w,   then the pairs of the first rot_dim columns turned by the token's position.

    wq, wk: float32 [d] or None (ones). table: rope_table(...), or None for the norm alone. q_positions, k_positions:
    int32 or int64 [N] or [B, N]; by default keys stand at 0 .. N_K - 1 and queries are the last N_Q of these places,
    as everywhere in this library. A side's default does not follow positions that are given for the other: with
    k_positions alone, queries still stand at N_K - N_Q .. N_K - 1. Places by default have to be in the table; a
    position given that is outside it gives NaN in the rotated columns, and no gradient where the loss does not reach
    the row (padding). interleaved: pairs (2j, 2j + 1) instead of (j, j + rot_dim/2). expand_k: write every key head
    once per query head of its group, so that yk has H heads (the gradients of the copies are added).
    """
    if _differentiated(q, k, wq, wk, table):
        if table is not None and table.requires_grad and torch.is_grad_enabled():
            raise ValueError("the table takes no gradient: pass it detached")
        return _QKNormRope.apply(q, k, wq, wk, table, float(eps), q_positions, k_positions, bool(interleaved),
                                 bool(expand_k))
    return qk_norm_rope_fwd(q, k, wq, wk, table, eps, q_positions, k_positions, interleaved, expand_k)


class QKPrep(typing.NamedTuple):
    """How the projections of one side become its queries and keys: the arguments of qk_norm_rope."""
    wq: torch.Tensor | None = None
    wk: torch.Tensor | None = None
    table: torch.Tensor | None = None
    eps: float = 1e-6
    interleaved: bool = False


def attention_kl_proj(q1, k1, q2, k2, prep1=QKPrep(), prep2=QKPrep(), *, q_positions=None, k_positions=None, **kl):
    """attention_kl from the projections of both sides, before norm and rotation.

    q1, q2 [B, N_Q, H, d_t] and k1, k2 [B, N_K, HK_t, d_t] as qk_norm_rope takes them (H a multiple of each side's
    HK_t; shared key heads are written once per query head). prep1, prep2: QKPrep of the sides. Positions are shared by
    them. The other options are attention_kl's. Gradients reach the projections and the norms' weights that require them.
    """
    sides = []
    for q, k, p in ((q1, k1, prep1), (q2, k2, prep2)):
        sides += qk_norm_rope(q, k, p.wq, p.wk, p.table, eps=p.eps, q_positions=q_positions, k_positions=k_positions,
                              interleaved=p.interleaved, expand_k=True)
    return attention_kl(*sides, **kl)


# --- differential attention -------------------------------------------------------------------------------------------


def _diff_error(q1, k1, q2, k2, v):
    """What is wrong with the tensors of a differential-attention call."""
    for n, t in (("q1", q1), ("k1", k1), ("q2", q2), ("k2", k2), ("v", v)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            return ValueError(f"{n} must be a GPU tensor")
        if t.dtype != torch.bfloat16:
            return ValueError(f"{n} must be bfloat16, got {t.dtype}")
        if t.dim() != 4:
            return ValueError(f"{n} must be a [B, H, N, d] tensor")
    if len({t.device for t in (q1, k1, q2, k2, v)}) != 1:
        return ValueError("all inputs must be on one device")
    return ValueError(f"inconsistent shapes q1{tuple(q1.shape)} k1{tuple(k1.shape)} q2{tuple(q2.shape)} "
                      f"k2{tuple(k2.shape)} v{tuple(v.shape)}")


def _diff_inputs(q1, k1, q2, k2, v, lam, q_len, kv_len):
    """Checked extents of the differential-attention calls: (device, (B, H, HK, N_Q, N_K, d, dv))."""
    for t in (q1, k1, q2, k2, v):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.bfloat16 and t.dim() == 4):
            raise _diff_error(q1, k1, q2, k2, v)
    dev, qs, ks = q1.device, q1.shape, k1.shape
    B, H, NQ, d = qs
    kb, HK, NK, kd = ks
    vb, vh, vn, dv = v.shape
    if q2.shape != qs or k2.shape != ks or kb != B or kd != d or vb != B or vh != HK or vn != NK or \
            k1.device != dev or q2.device != dev or k2.device != dev or v.device != dev:
        raise _diff_error(q1, k1, q2, k2, v)
    if NQ > _MAX_INT or NK > _MAX_INT or B > _MAX_INT or H > _MAX_INT:
        raise ValueError("an extent does not fit 31 bits")
    if (HK == 0) != (H == 0) or (HK and H % HK):
        raise ValueError(f"{H} query heads do not share {HK} key heads evenly")
    if not (isinstance(lam, torch.Tensor) and lam.dtype is torch.float32 and lam.shape == (H,) and
            lam.is_contiguous() and lam.device == dev):
        raise ValueError(f"lam must be a contiguous float32 tensor of shape {(H,)} on {dev}")
    for n, t in (("q_len", q_len), ("kv_len", kv_len)):
        if t is not None and (t.dtype != torch.int32 or t.shape != (B,) or not t.is_contiguous() or t.device != dev):
            raise ValueError(f"{n} must be a contiguous int32 tensor of shape {(B,)} on {dev}")
    return dev, (B, H, HK, NQ, NK, d, dv)


def _diff_scale(scale, d):
    return 1.0 / math.sqrt(d) if scale is None else float(scale)


def diff_split_count(B, H, HK, n_q, n_k, d, dv, causal=False) -> int:
    """streamkl_diff_fwd_split_count: the library's choice of splits (0 for invalid arguments)."""
    return int(lib.streamkl_diff_fwd_split_count(int(B), int(H), int(HK), int(n_q), int(n_k), int(d), int(dv),
                                                 int(bool(causal))))


def diff_workspace_bytes(B, H, n_q, dv, splits) -> int:
    """streamkl_diff_fwd_workspace_bytes: workspace of the split forward."""
    return int(lib.streamkl_diff_fwd_workspace_bytes(int(B), int(H), int(n_q), int(dv), int(splits)))


def diff_bwd_workspace_bytes(B, H, HK, n_q, n_k, d, dv, causal) -> int:
    """streamkl_diff_bwd_workspace_bytes: workspace of the backward."""
    return int(lib.streamkl_diff_bwd_workspace_bytes(int(B), int(H), int(HK), int(n_q), int(n_k), int(d), int(dv),
                                                     int(bool(causal))))


def diff_fwd(q1, k1, q2, k2, v, lam, scale=None, causal=False, q_len=None, kv_len=None, splits="auto", save=False,
             out=None, workspace=None):
    """streamkl_diff_fwd: the output, bf16 [B, H, N_Q, dv], or with ``save`` (out, out2, lse1, lse2), what diff_bwd
    needs. See diff_attention. splits: an int >= 1 or "auto" (diff_split_count). ``out`` may be a preallocated output;
    the split workspace is allocated here unless ``workspace`` (diff_workspace_bytes) is given."""
    dev, ext = _diff_inputs(q1, k1, q2, k2, v, lam, q_len, kv_len)
    B, H, HK, NQ, NK, d, dv = ext
    n = lib.streamkl_diff_fwd_split_count(*ext, int(bool(causal))) or 1 if splits == "auto" else int(splits)
    out = _bf16_out(out, (B, H, NQ, dv), dev, "out")
    out2 = lse1 = lse2 = None
    if save:
        out2 = torch.empty((B, H, NQ, dv), dtype=torch.bfloat16, device=dev)
        lse1, lse2 = torch.empty((2, B, H, NQ), dtype=torch.float32, device=dev).unbind(0)
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = _workspace(workspace, dev)
    elif n > 1:
        ws_bytes = lib.streamkl_diff_fwd_workspace_bytes(B, H, NQ, dv, n)
        workspace = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=dev)
    with _on(dev):
        st = lib.streamkl_diff_fwd(_rows(q1, "q1"), _rows(k1, "k1"), _rows(q2, "q2"), _rows(k2, "k2"), _rows(v, "v"),
                                   *ext, _diff_scale(scale, d), int(bool(causal)), _p(lam), _p(q_len), _p(kv_len), n,
                                   _p(workspace), ws_bytes, _p(out), _p(out2), _p(lse1), _p(lse2), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_diff_fwd")
    return (out, out2, lse1, lse2) if save else out


DIFF_GRADS = ("dq1", "dk1", "dq2", "dk2", "dv", "dlam")


def diff_bwd(q1, k1, q2, k2, v, lam, dout, out, out2, lse1, lse2, scale=None, causal=False, q_len=None, kv_len=None,
             want=DIFF_GRADS, grad_dtype=torch.float32, workspace=None):
    """streamkl_diff_bwd: (dq1, dk1, dq2, dk2, dv, dlam), None where not in ``want``; from dout (bf16, contiguous) and
    the results of diff_fwd(..., save=True). grad_dtype: float32 or bfloat16 (dlam is float32 always)."""
    dev, ext = _diff_inputs(q1, k1, q2, k2, v, lam, q_len, kv_len)
    B, H, HK, NQ, NK, d, dv = ext
    unknown = set(want) - set(DIFF_GRADS)
    if unknown or not want:
        raise ValueError(f"want must name some of {DIFF_GRADS}, got {sorted(want)}")
    if grad_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"grad_dtype must be float32 or bfloat16, got {grad_dtype}")
    for n, t in (("dout", dout), ("out", out), ("out2", out2)):
        if t is None:
            raise ValueError(f"{n} is missing")
        _bf16_out(t, (B, H, NQ, dv), dev, n)
    for n, t in (("lse1", lse1), ("lse2", lse2)):
        if t is None:
            raise ValueError(f"{n} is missing")
        _f32_rows(t, (B, H, NQ), dev, n)
    shapes = {"dq1": (B, H, NQ, d), "dk1": (B, HK, NK, d), "dq2": (B, H, NQ, d), "dk2": (B, HK, NK, d),
              "dv": (B, HK, NK, dv), "dlam": (H,)}
    g = {n: torch.empty(s, dtype=torch.float32 if n == "dlam" else grad_dtype, device=dev) if n in want else None
         for n, s in shapes.items()}
    if workspace is None:
        ws_bytes = lib.streamkl_diff_bwd_workspace_bytes(*ext, int(bool(causal)))
        workspace = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=dev)
    else:
        ws_bytes = _workspace(workspace, dev)
    with _on(dev):
        st = lib.streamkl_diff_bwd(_rows(q1, "q1"), _rows(k1, "k1"), _rows(q2, "q2"), _rows(k2, "k2"), _rows(v, "v"),
                                   *ext, _diff_scale(scale, d), int(bool(causal)), _p(lam), _p(q_len), _p(kv_len),
                                   _p(dout), _p(out), _p(out2), _p(lse1), _p(lse2), _p(workspace), ws_bytes,
                                   *(_p(g[n]) for n in DIFF_GRADS), int(grad_dtype == torch.bfloat16), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_diff_bwd")
    return tuple(g[n] for n in DIFF_GRADS)


class _DiffAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q1, k1, q2, k2, v, lam, scale, causal, q_len, kv_len):
        saved = diff_fwd(q1, k1, q2, k2, v, lam, scale, causal, q_len, kv_len, save=True)
        ctx.save_for_backward(q1, k1, q2, k2, v, lam, q_len, kv_len, *saved)
        ctx.cfg = (scale, causal)
        return saved[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q1, k1, q2, k2, v, lam, q_len, kv_len, *saved = ctx.saved_tensors
        scale, causal = ctx.cfg
        want = tuple(n for n, need in zip(DIFF_GRADS, ctx.needs_input_grad) if need)
        if not want:
            return (None,) * 10
        grads = diff_bwd(q1, k1, q2, k2, v, lam, _upstream(dout.to(torch.bfloat16)), *saved, scale, causal, q_len,
                         kv_len, want=want, grad_dtype=torch.bfloat16)
        return (*grads, None, None, None, None)


def diff_attention(q1, k1, q2, k2, v, lam, *, scale=None, causal=False, q_len=None, kv_len=None):
    """Differential attention, (softmax(scale q1 k1^T) - lam_h softmax(scale q2 k2^T)) v, differentiable.

    q1, q2 [B, H, N_Q, d], k1, k2 [B, HK, N_K, d], v [B, HK, N_K, dv], bf16 with contiguous 16-byte aligned rows in any
    arrangement (halves of one projection, values as their projection leaves them, the filled part of a cache). H is a
    multiple of HK: groups of H / HK query heads share keys and values. lam float32 [H]. Returns bf16 [B, H, N_Q, dv],
    contiguous; gradients come in the inputs' types.

    causal: bottom-right alignment, as everywhere in this library. q_len, kv_len: int32 [B] on the device; sequence b
    has its first q_len[b] rows and kv_len[b] keys (a right-padded batch, caches filled to different lengths). Rows
    behind q_len and rows that see no key give 0. scale defaults to 1/sqrt(d).

    To capture a training step into a HIP graph, capture it while no eager graph of the same leaves is alive (drop the
    warm-up's outputs first): autograd's accumulation nodes of an eager graph belong to its stream, and torch ends the
    process where a captured backward meets them. The same holds for the other autograd
    functions here.
    """
    scale = _diff_scale(scale, q1.shape[-1])
    if _differentiated(q1, k1, q2, k2, v, lam):
        return _DiffAttention.apply(q1, k1, q2, k2, v, lam, scale, bool(causal), q_len, kv_len)
    return diff_fwd(q1, k1, q2, k2, v, lam, scale, causal, q_len, kv_len)


# --- rows of logits: log probabilities, entropies, best tokens --------------------------------------------------------


class TokenLogprobs(typing.NamedTuple):
    """What token_logprobs returns; None where not asked for."""
    logp: torch.Tensor | None
    entropy: torch.Tensor | None
    lse: torch.Tensor
    top_logp: torch.Tensor | None
    top_ids: torch.Tensor | None


def _logit_error(t, name):
    """What is wrong with a tensor of logits."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        return ValueError(f"{name} must be a GPU tensor")
    if t.dtype not in DTYPES:
        return ValueError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
    if t.dim() not in (2, 3):
        return ValueError(f"{name} must be a [N, V] or [B, N, V] tensor, got {tuple(t.shape)}")
    return ValueError(f"{name} must be contiguous along its last axis")


def _logits(t, name="logits"):
    """A tensor of logits as a streamkl_logits: (device, shape of its rows, V, streamkl_logits)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in DTYPES and t.dim() in (2, 3)):
        raise _logit_error(t, name)
    shape, st = t.shape, t.stride()
    V = shape[-1]
    if st[-1] != 1 and V != 1:
        raise _logit_error(t, name)
    B, N = (1, shape[0]) if len(shape) == 2 else shape[:2]
    if B > _MAX_INT or N > _MAX_INT or V > _MAX_INT:
        raise ValueError("an extent does not fit 31 bits")
    # the stride of an extent of one says nothing
    sb = st[0] if len(shape) == 3 and B > 1 else 0
    return t.device, shape[:-1], V, _Logits(t.data_ptr(), sb, st[-2] if N > 1 else 0, B, N, V, DTYPES[t.dtype])


def _ints(t, shape, dev, name):
    if not (isinstance(t, torch.Tensor) and t.dtype in (torch.int32, torch.int64) and t.shape == shape and
            t.is_contiguous() and t.device == dev):
        raise ValueError(f"{name} must be a contiguous int32 or int64 tensor of shape {tuple(shape)} on {dev}")
    return int(t.dtype is torch.int64)


def _row_floats(t, shape, dev, name):
    if t is not None and not (isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.shape == shape and
                              t.is_contiguous() and t.device == dev):
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape {tuple(shape)} on {dev}")
    return t


def _grad_rows(out, logits):
    """A tensor for the gradient of the logits, new or the caller's: (tensor, strides between sequences and rows)."""
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif not (isinstance(out, torch.Tensor) and out.dtype == logits.dtype and out.shape == logits.shape and
              out.device == logits.device):
        raise ValueError(f"out must be a {logits.dtype} tensor of shape {tuple(logits.shape)} on {logits.device}")
    _, _, _, rows = _logits(out, "out")
    return out, rows.sb, rows.sn


def token_logprobs_workspace_bytes(B, N, V, dtype, top=0) -> int:
    """streamkl_token_logprobs_workspace_bytes."""
    return int(lib.streamkl_token_logprobs_workspace_bytes(int(B), int(N), int(V), DTYPES[dtype], int(top)))


def token_logprobs_fwd(logits, tokens=None, scale=1.0, top=0, entropy=True, save=False, workspace=None):
    """streamkl_token_logprobs_fwd: TokenLogprobs, with ``save`` also lse_err, which token_logprobs_bwd takes. See
    token_logprobs. The workspace (16-byte aligned) is allocated here unless given."""
    dev, shape, V, rows = _logits(logits)
    tokens64 = 0 if tokens is None else _ints(tokens, shape, dev, "tokens")
    top = int(top)
    if not 0 <= top <= V:
        raise ValueError(f"top must be 0 to the vocabulary's {V}, got {top}")
    # the rows' numbers from one allocation (1.5 us each), but each a tensor of its own (.data): of views autograd would refuse
    # to edit one in place, or take the others for edited
    want = (True, tokens is not None, bool(entropy), save)
    made = iter(torch.empty((sum(want), *shape), dtype=torch.float32, device=dev).unbind(0))
    lse, logp, ent, err = (next(made).data if w else None for w in want)
    top_logp = top_ids = None
    if top:
        top_logp = torch.empty((*shape, top), dtype=torch.float32, device=dev)
        top_ids = torch.empty((*shape, top), dtype=torch.int32, device=dev)
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = _workspace(workspace, dev)
    elif top <= 128:
        ws_bytes = lib.streamkl_token_logprobs_workspace_bytes(rows.B, rows.N, V, rows.dtype, top)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        st = lib.streamkl_token_logprobs_fwd(rows, _p(tokens), tokens64, float(scale), top, _p(workspace), ws_bytes,
                                             _p(logp), _p(ent), _p(lse), _p(err), _p(top_logp), _p(top_ids), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_token_logprobs_fwd")
    y = TokenLogprobs(logp, ent, lse, top_logp, top_ids)
    return (y, err) if save else y


def token_logprobs_bwd(logits, tokens, lse, lse_err=None, entropy=None, dlogp=None, dentropy=None, dlse=None, scale=1.0,
                       out=None):
    """streamkl_token_logprobs_bwd: the gradient of the logits, in their type. lse, lse_err and entropy are those of
    token_logprobs_fwd(..., save=True). ``out`` may be a tensor of the logits' shape and type with rows that do not
    overlap, the logits themselves among them."""
    dev, shape, _, rows = _logits(logits)
    tokens64 = 0 if tokens is None else _ints(tokens, shape, dev, "tokens")
    if lse is None:
        raise ValueError("lse is missing")
    args = [_p(_row_floats(t, shape, dev, n)) for n, t in
            (("lse", lse), ("lse_err", lse_err), ("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy),
             ("dlse", dlse))]
    if dlogp is not None and tokens is None:
        raise ValueError("dlogp given without tokens")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy given without entropy")
    out, sb, sn = _grad_rows(out, logits)
    with _on(dev):
        st = lib.streamkl_token_logprobs_bwd(rows, _p(tokens), tokens64, float(scale), *args, _p(out), sb, sn,
                                             _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_token_logprobs_bwd")
    return out


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, scale, top, entropy):
        y, err = token_logprobs_fwd(logits, tokens, scale, top, entropy, save=True)
        ctx.save_for_backward(logits, tokens, y.lse, err, y.entropy)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        if top:
            ctx.mark_non_differentiable(y.top_logp, y.top_ids)
        return tuple(y)

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dentropy, dlse, _top, _ids):
        logits, tokens, lse, err, entropy = ctx.saved_tensors
        up = [None if g is None else g.to(torch.float32).contiguous() for g in (dlogp, dentropy, dlse)]
        if all(g is None for g in up):
            return (None,) * 5
        return (token_logprobs_bwd(logits, tokens, lse, err, entropy, *up, ctx.scale), None, None, None, None)


def token_logprobs(logits, tokens=None, *, scale=1.0, top=0, entropy=True):
    """Log probabilities of given tokens under softmax(scale logits), with entropies and the best tokens; differentiable.

    logits [N, V] or [B, N, V] in bfloat16, float16 or float32, rows anywhere in memory (a vocabulary of any size, a slice
    of a padded one, logits[:, :-1]). tokens: int32 or int64 [N] or [B, N], or None; a negative token is none (padding)
    and has logp 0, one outside the vocabulary NaN (and NaN gradients where logp has an upstream gradient). scale: an
    inverse temperature. top: 0 to 128.

    Returns TokenLogprobs: logp, entropy (nats; None unless ``entropy``) and lse = log sum exp(scale logits), float32 of
    the tokens' shape; top_logp (float32) and top_ids (int32) [..., top], descending, the lowest index first among equal
    logits. Gradients flow through logp, entropy and lse in the logits' type. Logits of -inf have probability 0; a row
    of nothing else has lse -inf, entropy 0 and no gradient.
    """
    if _differentiated(logits):
        return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, float(scale), int(top), bool(entropy)))
    return token_logprobs_fwd(logits, tokens, scale, top, entropy)


# --- distillation from a teacher's best tokens ------------------------------------------------------------------------


def _distill_inputs(logits, ids, teacher, s1, s2, rest, direction):
    """Checked arguments of the distillation calls: (device, shape of the rows, arguments that all calls begin with)."""
    dev, shape, V, rows = _logits(logits)
    if not (isinstance(ids, torch.Tensor) and ids.dim() == logits.dim()):
        raise ValueError(f"ids must be a tensor of shape {(*shape, 'K')}")
    lists = (*shape, ids.shape[-1])
    ids64 = _ints(ids, lists, dev, "ids")
    if not (isinstance(teacher, torch.Tensor) and teacher.dtype in DTYPES and teacher.shape == lists and
            teacher.is_contiguous() and teacher.device == dev):
        raise ValueError(f"teacher must be a contiguous bfloat16, float16 or float32 tensor of shape {lists} on {dev}")
    d = _direction(direction)
    if rest and s1 != 1.0:
        raise ValueError("s1 must be 1 with a rest: that of a distribution at another temperature is not known")
    if d == REV and not rest:
        raise ValueError("the reverse direction needs a rest: a student's tokens outside the list have no teacher")
    listed = _TeacherList(ids.data_ptr(), teacher.data_ptr(), lists[-1], ids64, DTYPES[teacher.dtype], int(bool(rest)),
                          float(s1))
    return dev, shape, (rows, listed, float(s2), d)


def topk_distill_workspace_bytes(B, N, V, dtype, rest=True) -> int:
    """streamkl_topk_distill_workspace_bytes."""
    return int(lib.streamkl_topk_distill_workspace_bytes(int(B), int(N), int(V), DTYPES[dtype], int(bool(rest))))


def _distill_workspace(workspace, dev, args):
    if workspace is not None:
        return workspace, _workspace(workspace, dev)
    rows, listed = args[:2]
    n = lib.streamkl_topk_distill_workspace_bytes(rows.B, rows.N, rows.V, rows.dtype, listed.rest)
    return (torch.empty(n, dtype=torch.uint8, device=dev) if n else None), n


def _distill_stats(stats, shape, dev):
    if not (isinstance(stats, torch.Tensor) and stats.dtype is torch.float64 and stats.shape == (*shape, 4) and
            stats.is_contiguous() and stats.device == dev):
        raise ValueError(f"stats must be a contiguous float64 tensor of shape {(*shape, 4)} on {dev}")
    return stats


def topk_distill_fwd(logits, ids, teacher, s1=1.0, s2=1.0, rest=True, direction=FWD, workspace=None):
    """streamkl_topk_distill_fwd: (loss, stats), float32 of the rows' shape and what topk_distill_bwd needs (float64
    [..., 4]). See topk_distill. The workspace (16-byte aligned) is allocated here unless given."""
    dev, shape, args = _distill_inputs(logits, ids, teacher, s1, s2, rest, direction)
    loss = torch.empty(shape, dtype=torch.float32, device=dev)
    stats = torch.empty((*shape, 4), dtype=torch.float64, device=dev)
    workspace, ws_bytes = _distill_workspace(workspace, dev, args)
    with _on(dev):
        st = lib.streamkl_topk_distill_fwd(*args, _p(workspace), ws_bytes, _p(loss), _p(stats), _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_topk_distill_fwd")
    return loss, stats


def topk_distill_bwd(logits, ids, teacher, stats, dloss=None, s1=1.0, s2=1.0, rest=True, direction=FWD, factor=1.0,
                     dfactor=None, done_if_one=False, out=None):
    """streamkl_topk_distill_bwd: the gradient of the logits, in their type, for the upstream gradients
    dloss (float32 of the rows' shape, None: ones) times factor times dfactor (a float32 tensor of one element, None: 1).
    done_if_one: ``out`` already holds it for dfactor 1 (topk_distill_step) and is left alone then. ``out`` may be a
    tensor of the logits' shape and type with rows that do not overlap, the logits themselves among them (but with
    done_if_one, where it holds the gradient)."""
    dev, shape, args = _distill_inputs(logits, ids, teacher, s1, s2, rest, direction)
    _distill_stats(stats, shape, dev)
    _row_floats(dloss, shape, dev, "dloss")
    if dfactor is not None and not (dfactor.dtype is torch.float32 and dfactor.numel() == 1 and dfactor.device == dev):
        raise ValueError(f"dfactor must be a float32 tensor of one element on {dev}")
    if done_if_one and (out is None or dfactor is None):
        raise ValueError("done_if_one needs out and dfactor")
    if done_if_one and out.data_ptr() == logits.data_ptr() and out.numel():
        raise ValueError("out holds the gradient with done_if_one: the logits must be elsewhere")
    out, sb, sn = _grad_rows(out, logits)
    with _on(dev):
        st = lib.streamkl_topk_distill_bwd(*args, _p(stats), _p(dloss), float(factor), _p(dfactor),
                                           int(bool(done_if_one)), _p(out), sb, sn, _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_topk_distill_bwd")
    return out


def topk_distill_step(logits, ids, teacher, weight=None, s1=1.0, s2=1.0, rest=True, direction=FWD, factor=1.0, out=None,
                      workspace=None):
    """streamkl_topk_distill_step: (loss, stats, dlogits), the rows' losses with the gradient of
    sum(weight * factor * loss). weight: float32 of the rows' shape, None: ones. Others as in topk_distill_fwd and
    topk_distill_bwd."""
    dev, shape, args = _distill_inputs(logits, ids, teacher, s1, s2, rest, direction)
    _row_floats(weight, shape, dev, "weight")
    loss = torch.empty(shape, dtype=torch.float32, device=dev)
    stats = torch.empty((*shape, 4), dtype=torch.float64, device=dev)
    workspace, ws_bytes = _distill_workspace(workspace, dev, args)
    out, sb, sn = _grad_rows(out, logits)
    with _on(dev):
        st = lib.streamkl_topk_distill_step(*args, _p(workspace), ws_bytes, _p(weight), float(factor), _p(loss),
                                            _p(stats), _p(out), sb, sn, _stream(dev))
    if st != OK:
        raise StreamKLError(st, "streamkl_topk_distill_step")
    return loss, stats, out


def _distill_total(loss, weight, factor):
    total = torch.empty((), dtype=torch.float32, device=loss.device)
    with _on(loss.device):
        st = lib.streamkl_topk_distill_total(_p(loss), _p(weight), factor, loss.numel(), _p(total), _stream(loss.device))
    if st != OK:
        raise StreamKLError(st, "streamkl_topk_distill_total")
    return total


class _TopkDistill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, opts):
        loss, stats = topk_distill_fwd(logits, ids, teacher, *opts)
        ctx.save_for_backward(logits, ids, teacher, stats)
        ctx.opts = opts
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        logits, ids, teacher, stats = ctx.saved_tensors
        return (topk_distill_bwd(logits, ids, teacher, stats, dloss.to(torch.float32).contiguous(), *ctx.opts),
                None, None, None)


class _TopkDistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, weight, factor, opts):
        loss, stats, grad = topk_distill_step(logits, ids, teacher, weight, *opts, factor)
        # grad, for an upstream gradient of 1, among the tensors that hooks on saved tensors (offloading, checkpoints) see
        ctx.save_for_backward(logits, ids, teacher, weight, stats, grad)
        ctx.cfg = (factor, opts)
        ctx.handed_over = False
        return _distill_total(loss, weight, factor)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        logits, ids, teacher, weight, stats, grad = ctx.saved_tensors
        factor, opts = ctx.cfg
        # the first backward pass hands the gradient over; a later one through a retained graph forms it again. As a tensor
        # of its own (.data): the saved one does not see what becomes of it, and a leaf takes it without a copy
        out = None if ctx.handed_over else grad.data
        ctx.handed_over = True
        del grad
        return (topk_distill_bwd(logits, ids, teacher, stats, weight, *opts, factor, g.to(torch.float32), out is not None,
                                 out), None, None, None, None, None)


def _no_gradient(**tensors):
    if torch.is_grad_enabled():
        for n, t in tensors.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{n} takes no gradient: pass it detached")


def topk_distill(logits, ids, teacher, *, s1=1.0, s2=1.0, rest=True, direction="fwd"):
    """Per-row divergence of a student, softmax(s2 logits) over the vocabulary, from a teacher's best tokens;
    differentiable in the logits.

    logits [N, V] or [B, N, V] as token_logprobs takes them. ids (int32 or int64) and teacher (float32, bfloat16 or
    float16) [..., K], K up to 128: the teacher's tokens of every row and their values, such as top_ids and top_logp of
    token_logprobs. A negative id is no entry: lists may be of unequal length, a row without entries has no loss.

    rest=True: the values are natural log probabilities, and the mass outside the list is one bucket of both
    distributions. direction "fwd" is KL(teacher || student), "rev" KL(student || teacher), as in attention_kl.
    rest=False: the list is all the teacher has, softmax(s1 teacher) over it; "fwd" only.

    Returns float32 losses of the rows' shape; the gradient comes in the logits' type. For a weighted sum of the rows
    topk_distill_loss is faster: it reads the logits once.
    """
    opts = (s1, s2, rest, direction)
    if _differentiated(logits, teacher):
        _no_gradient(teacher=teacher)
        return _TopkDistill.apply(logits, ids, teacher, opts)
    return topk_distill_fwd(logits, ids, teacher, *opts)[0]


def topk_distill_loss(logits, ids, teacher, weight=None, *, s1=1.0, s2=1.0, rest=True, direction="fwd"):
    """sum(weight * topk_distill(logits, ids, teacher, ...)), a scalar; weight float32 of the rows' shape, or None for the
    mean over all rows. Rows of weight 0 (padding) are left out, whatever they hold.

    The weights are known before the losses, so the gradient is formed with them, in the forward call where the logits
    require one (memory of the logits' size from there on, saved as autograd saves tensors: hooks on these see it, and a
    checkpoint keeps none of it). The backward pass hands it over; for an upstream gradient other than 1 (a loss scale) it
    forms the gradient anew, rounded once. Under torch.no_grad() only the loss is formed.
    """
    opts = (s1, s2, rest, direction)
    rows = logits.numel() // logits.shape[-1] if isinstance(logits, torch.Tensor) and logits.numel() else 0
    factor = 1.0 if weight is not None else 1.0 / max(rows, 1)
    if _differentiated(logits, teacher, weight):
        _no_gradient(teacher=teacher, weight=weight)
        return _TopkDistillLoss.apply(logits, ids, teacher, weight, factor, opts)
    loss = topk_distill_fwd(logits, ids, teacher, *opts)[0]
    return _distill_total(loss, _row_floats(weight, loss.shape, loss.device, "weight"), factor)
