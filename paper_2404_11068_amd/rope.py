"""Python binding of the C ABI in include/evo_rope.h (argument marshalling only),
and the tables of frequencies that the calls take.

Rotary positions, and the norm of every head with the rotation in the same
pass, run in ``libevoattn.so``; this module passes torch tensors' device
pointers and raises on a nonzero status.  No fallback exists.

  q, k : [N, Lq, H, d], [N, Lk, Hk, d] bf16 or fp32, the [H, d] block of each token contiguous;
      row and token strides are free (views of packed projections), lengths and heads of the two may differ
  pos_q, pos_k : int32 [N, L] or [1, L] or [L] (all rows the same), any values
  steps : int64 [rot / 2] from rope_steps: turns per position in units of 2^-64; rot <= d channels are rotated
  weight_q, weight_k : fp32 [d] or None (ones)
"""
from __future__ import annotations

import ctypes
import math
from fractions import Fraction
from typing import List, Optional, Tuple

import torch

from .evo_attn import EvoAttnError, _DTYPES, _empty, _stream, load_library

_INTERLEAVED, _NORM = 1, 2


class evo_rope_dims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("n_heads", ctypes.c_int32 * 2), ("eps", ctypes.c_float),
                ("amplitude", ctypes.c_float), ("n_rows", ctypes.c_int64), ("len", ctypes.c_int64 * 2),
                ("pos_stride", ctypes.c_int64 * 2), ("x_stride_row", ctypes.c_int64 * 2),
                ("x_stride_tok", ctypes.c_int64 * 2), ("y_stride_row", ctypes.c_int64 * 2),
                ("y_stride_tok", ctypes.c_int64 * 2)]


_bound = False


def _lib():
    global _bound
    lib = load_library()
    if not _bound:
        P = ctypes.c_void_p
        D = ctypes.POINTER(evo_rope_dims)
        lib.evo_rope_fwd.argtypes = [D] + [P] * 10
        lib.evo_rope_fwd.restype = ctypes.c_int
        lib.evo_rope_bwd_workspace_size.argtypes = [D]
        lib.evo_rope_bwd_workspace_size.restype = ctypes.c_size_t
        lib.evo_rope_bwd.argtypes = [D] + [P] * 14 + [ctypes.c_size_t, P]
        lib.evo_rope_bwd.restype = ctypes.c_int
        _bound = True
    return lib


# 1 / (2 pi) to 60 decimals: 2^-64 of a turn is 19 of them
_PER_RADIAN = Fraction(159154943091895335768883763372514362034459645740456448747667, 10 ** 60)


def rope_frequencies(rot_dim: int, base: float = 10000.0, *, factor: float = 1.0, scaling: str = "linear",
                     trained_length: int = 4096, fast: float = 32.0, slow: float = 1.0) -> List[float]:
    """Radians per position of the rot_dim / 2 pairs, base^(-2i / rot_dim), for contexts `factor` times as long:

    "linear": all frequencies divided by factor (positions interpolated).
    "base": a base larger by factor^(rot_dim / (rot_dim - 2)): the last pair is divided by factor, the first kept.
    "turns": pairs that make `fast` turns or more over trained_length keep their frequency, those that make
        `slow` or fewer have it divided, between them the share kept runs along the logarithm of the turns;
        rope_amplitude(factor) goes with it.
    """
    if rot_dim < 0 or rot_dim % 2 or not base > 0 or not factor > 0:
        raise ValueError("rot_dim must be even and not negative, base and factor positive")
    if scaling not in ("linear", "base", "turns"):
        raise ValueError('scaling must be "linear", "base" or "turns"')
    if scaling == "turns" and not (trained_length > 0 and fast > slow > 0):
        raise ValueError("trained_length must be positive and fast > slow > 0")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    freq = [base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling == "linear":
        return [f / factor for f in freq]
    if scaling == "turns":
        keep = [math.log(trained_length * f / (2 * math.pi) / slow) / math.log(fast / slow) for f in freq]
        keep = [min(1.0, max(0.0, s)) for s in keep]
        return [f * (s + (1 - s) / factor) for f, s in zip(freq, keep)]
    return freq


def rope_amplitude(factor: float) -> float:
    """Amplitude that goes with "turns" scaling: 0.1 ln(factor) + 1, and 1 for factors up to 1."""
    return 1.0 if factor <= 1.0 else 0.1 * math.log(factor) + 1.0


def rope_steps(frequencies, device="cuda") -> torch.Tensor:
    """int64 [rot / 2]: each frequency (radians per position: a list, or a float tensor, which is read on the
    host) as turns per position times 2^64, modulo whole turns.  Laid out once; off by at most half of 2^-64
    turns, that is 2^-34 turns at position 2^31."""
    if isinstance(frequencies, torch.Tensor):
        device = frequencies.device
        frequencies = frequencies.double().tolist()
    steps = []
    for f in frequencies:
        if not math.isfinite(f):
            raise ValueError("frequencies must be finite")
        s = round(Fraction(f) * _PER_RADIAN * 2 ** 64) % 2 ** 64
        steps.append(s - 2 ** 64 if s >= 2 ** 63 else s)
    return torch.tensor(steps, dtype=torch.int64, device=device)


def _check_tokens(x: torch.Tensor, what: str, like: Optional[torch.Tensor] = None):
    if x.dim() != 4:
        raise ValueError("%s must be [N, L, H, d]" % what)
    if x.dtype not in _DTYPES:
        raise ValueError("%s must be float32 or bfloat16" % what)
    N, L, H, d = x.shape
    sr, st, sh, sd = x.stride()
    if (d > 1 and sd != 1) or (H > 1 and sh != d):
        raise ValueError("the [H, d] block of each token of %s must be contiguous" % what)
    if like is not None and (x.dtype != like.dtype or x.device != like.device or d != like.shape[3] or N != like.shape[0]):
        raise ValueError("%s must share its type, device, rows and head dim with the queries" % what)
    return N, L, H, d, (sr if N > 1 else 0), (st if L > 1 else 0)


def _strides(x: torch.Tensor, fill: bool):
    """(row, token) strides; of an axis of one entry, whose stride says nothing, the packed value."""
    N, L, H, d = x.shape
    tok = x.stride(1) if L > 1 else H * d
    row = x.stride(0) if N > 1 else (L * tok if fill else 0)
    return row, tok


def _check_pos(pos: Optional[torch.Tensor], N: int, L: int, like: torch.Tensor, what: str) -> int:
    """Checks; returns the positions' row stride."""
    if pos is None or pos.dtype != torch.int32 or pos.dim() not in (1, 2) or pos.shape[-1] != L or \
            (pos.dim() == 2 and pos.shape[0] not in (1, N)) or (L > 1 and pos.stride(-1) != 1):
        raise ValueError("%s must be int32 [%d, %d], [1, %d] or [%d] with contiguous rows" % (what, N, L, L, L))
    if pos.device != like.device:
        raise ValueError("tensors must be on one device")
    return pos.stride(0) if pos.dim() == 2 and pos.shape[0] > 1 else 0


def _check_weight(w: Optional[torch.Tensor], d: int, like: torch.Tensor, what: str):
    if w is not None and (w.dtype != torch.float32 or w.shape != (d,) or not w.is_contiguous() or w.device != like.device):
        raise ValueError("%s must be a contiguous float32 [%d] tensor on the queries' device" % (what, d))


def _dims(x, y, pos, steps, weights, interleaved, norm, eps, amplitude, pos_names=("pos_q", "pos_k")):
    """dims for the sets x (of dx, too) and y (of dy, too); also checks."""
    q = x[0]
    N, _, _, d, _, _ = _check_tokens(q, "q")
    if q.device.type != "cuda" or q.device.index != torch._C._cuda_getDevice():
        raise ValueError("tensors must be on the current CUDA device")
    if steps.dtype != torch.int64 or steps.dim() != 1 or not steps.is_contiguous() or steps.device != q.device:
        raise ValueError("steps must be a contiguous int64 [rot / 2] tensor on the queries' device")
    rot = 2 * steps.shape[0]
    if rot > d:
        raise ValueError("steps are for %d channels, a head has %d" % (rot, d))
    if not norm and (weights[0] is not None or weights[1] is not None):
        raise ValueError("weights go with norm=True")
    dm = evo_rope_dims()
    dm.dtype, dm.head_dim, dm.rot_dim, dm.n_rows = _DTYPES[q.dtype], d, rot, N
    dm.flags = (_INTERLEAVED if interleaved else 0) | (_NORM if norm else 0)
    dm.eps, dm.amplitude = eps, amplitude
    for i in range(2):
        if x[i] is None:
            if pos[i] is not None or weights[i] is not None:
                raise ValueError("%s and a weight for keys go with keys" % pos_names[i])
            continue
        _, L, H, _, _, _ = _check_tokens(x[i], "qk"[i], q)
        if y[i] is not None:
            _check_tokens(y[i], "gradient or output", q)
            if y[i].shape != x[i].shape:
                raise ValueError("outputs and gradients must be shaped like their heads")
        dm.n_heads[i], dm.len[i] = H, L
        dm.pos_stride[i] = _check_pos(pos[i], N, L, q, pos_names[i])
        _check_weight(weights[i], d, q, "weight")
        dm.x_stride_row[i], dm.x_stride_tok[i] = _strides(x[i], True)
        dm.y_stride_row[i], dm.y_stride_tok[i] = _strides(y[i], True) if y[i] is not None else (L * H * d, H * d)
    return dm


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def rope_fwd(q: torch.Tensor, pos_q: torch.Tensor, steps: torch.Tensor, *, k: Optional[torch.Tensor] = None,
             pos_k: Optional[torch.Tensor] = None, interleaved: bool = False, norm: bool = False,
             weight_q: Optional[torch.Tensor] = None, weight_k: Optional[torch.Tensor] = None, eps: float = 1e-6,
             amplitude: float = 1.0, out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None,
             stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rotated queries and keys (keys optional), with norm=True of every head over its root mean square, times the
    weight, first.  Pairs are (i, i + rot / 2), or (2i, 2i + 1) when interleaved; amplitude scales the rotated
    channels.  out_q=q, out_k=k work in place.  Returns (out_q, out_k or None)."""
    lib = _lib()
    dm = _dims((q, k), (out_q, out_k), (pos_q, pos_k), steps, (weight_q, weight_k), interleaved, norm, eps, amplitude)
    if k is None and out_k is not None:
        raise ValueError("out_k goes with k")
    if out_q is None:
        out_q = _empty(q.shape, q.dtype, q, stream)
    if k is not None and out_k is None:
        out_k = _empty(k.shape, k.dtype, q, stream)
    st = lib.evo_rope_fwd(dm, q.data_ptr(), _addr(k), _addr(pos_q), _addr(pos_k), steps.data_ptr(), _addr(weight_q),
                          _addr(weight_k), out_q.data_ptr(), _addr(out_k), _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_rope_fwd")
    return out_q, out_k


def rope_bwd_workspace_size(q: torch.Tensor, steps: torch.Tensor, *, k: Optional[torch.Tensor] = None,
                            norm: bool = False) -> int:
    """Bytes of workspace that rope_bwd needs for heads shaped like q and k."""
    dm = evo_rope_dims()
    N, _, _, d, _, _ = _check_tokens(q, "q")
    dm.dtype, dm.head_dim, dm.rot_dim, dm.n_rows = _DTYPES[q.dtype], d, 2 * steps.numel(), N
    dm.flags, dm.amplitude = (_NORM if norm else 0), 1.0
    for i, x in enumerate((q, k)):
        if x is not None:
            dm.len[i], dm.n_heads[i] = x.shape[1], x.shape[2]
            dm.x_stride_row[i], dm.x_stride_tok[i] = dm.y_stride_row[i], dm.y_stride_tok[i] = \
                x.shape[1] * x.shape[2] * d, x.shape[2] * d
    return int(_lib().evo_rope_bwd_workspace_size(dm))


def rope_bwd(dq: torch.Tensor, pos_q: torch.Tensor, steps: torch.Tensor, *, dk: Optional[torch.Tensor] = None,
             pos_k: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, k: Optional[torch.Tensor] = None,
             interleaved: bool = False, norm: bool = False, weight_q: Optional[torch.Tensor] = None,
             weight_k: Optional[torch.Tensor] = None, eps: float = 1e-6, amplitude: float = 1.0,
             out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None,
             dweight_q: Optional[torch.Tensor] = None, dweight_k: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of rope_fwd's queries and keys from dq, dk, those of its outputs; with norm=True q and k are
    rope_fwd's inputs.  out_q and out_k take the gradients (laid out like q and k where those are given; without
    the norm out_q=dq works in place).  Returns (gradient of q, of k, of weight_q, of weight_k), None for what
    is not there."""
    lib = _lib()
    if norm and (q is None or (k is None) != (dk is None)):
        raise ValueError("norm=True needs q, and k with dk")
    if not norm and (q is not None or k is not None):
        raise ValueError("q and k go with norm=True")
    if dk is None and out_k is not None:
        raise ValueError("out_k goes with dk")
    x = [q, k] if norm else [out_q, out_k]
    for i, (given, dy) in enumerate(((out_q, dq), (out_k, dk))):
        if dy is None:
            continue
        if norm and given is not None and (given.shape != x[i].shape or given.stride() != x[i].stride()):
            raise ValueError("out_q and out_k must be laid out like q and k")
        if x[i] is None:
            x[i] = _empty(dy.shape, dy.dtype, dq, stream)
    if (x[0].shape != dq.shape) or (dk is not None and x[1].shape != dk.shape):
        raise ValueError("gradients must be shaped like their heads")
    dm = _dims(x, (dq, dk), (pos_q, pos_k), steps, (weight_q, weight_k), interleaved, norm, eps, amplitude)
    outs = [out_q, out_k]
    for i, dy in enumerate((dq, dk)):
        if outs[i] is not None:
            if outs[i].dtype != dq.dtype or outs[i].device != dq.device:
                raise ValueError("out_q and out_k must share the gradients' type and device")
        elif dy is not None and not norm:
            outs[i] = x[i]
        elif dy is not None:
            t = x[i]
            if t.is_contiguous():
                outs[i] = _empty(t.shape, t.dtype, dq, stream)
            else:  # the layout of a view of packed projections: as large as what the view spans
                size = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1 if t.numel() else 0
                outs[i] = _empty((size,), t.dtype, dq, stream).as_strided(t.shape, t.stride())
    dws = [dweight_q, dweight_k]
    for i, w in enumerate((weight_q, weight_k)):
        if w is None:
            if dws[i] is not None:
                raise ValueError("a weight's gradient goes with the weight")
        elif dws[i] is None:
            dws[i] = _empty(w.shape, torch.float32, dq, stream)
        else:
            _check_weight(dws[i], w.shape[0], dq, "dweight")
    need = lib.evo_rope_bwd_workspace_size(dm)
    if workspace is None:
        ws_bytes, workspace = need, _empty((max(need, 1),), torch.uint8, dq, stream)
    elif workspace.device != dq.device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on the device of the gradients")
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    st = lib.evo_rope_bwd(dm, dq.data_ptr(), _addr(dk), _addr(x[0]) if norm else None, _addr(x[1]) if norm else None,
                          _addr(pos_q), _addr(pos_k), steps.data_ptr(), _addr(weight_q), _addr(weight_k),
                          outs[0].data_ptr(), _addr(outs[1]), _addr(dws[0]), _addr(dws[1]), workspace.data_ptr(),
                          ws_bytes, _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_rope_bwd")
    return outs[0], outs[1], dws[0], dws[1]
