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
    # (arrays of two as two fields each: they are set several times as fast)
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "head_dim", "rot_dim", "flags", "n_heads0", "n_heads1")] + \
        [("eps", ctypes.c_float), ("amplitude", ctypes.c_float), ("n_rows", ctypes.c_int64)] + \
        [(n + i, ctypes.c_int64) for n in ("len", "pos_stride", "x_stride_row", "x_stride_tok", "y_stride_row",
                                           "y_stride_tok") for i in "01"]


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
        `slow` or fewer have it divided, between them the share kept runs along the logarithm of the turns,
        which is along the pair's index, with bounds between whole pairs; rope_amplitude(factor) goes with it.
        A checkpoint of another ramp (linear in the turns, bounds rounded to whole pairs) has frequencies of
        its own, some of them by a third apart: give rope_steps that list.
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
    host) as turns per position times 2^64, modulo whole turns.  Laid out once (0.2 to 0.5 ms for 64 pairs on the
    host; not within a capture); off by at most half of 2^-64 turns, that is 2^-34 turns at position 2^31."""
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


def _layout(x: torch.Tensor, what: str):
    """(shape, row stride, token stride) of [N, L, H, d] heads; an axis of one entry, whose stride says nothing, counts
    as packed."""
    shape = x.shape
    if len(shape) != 4:
        raise ValueError("%s must be [N, L, H, d]" % what)
    N, L, H, d = shape
    row, tok, sh, sd = x.stride()
    if (sd != 1 and d > 1) or (sh != d and H > 1):
        raise ValueError("the [H, d] block of each token of %s must be contiguous" % what)
    if L <= 1:
        tok = H * d
    return shape, row if N > 1 and L > 0 else L * tok, tok


def _set(x, y, pos, w, q, what):
    """Checks of one set of heads x (of dx, too), with y (of dy, too; None: packed); what the dims say of it."""
    dtype, device = q.dtype, q.device
    shape, x_row, x_tok = _layout(x, what)
    N, L, H, d = shape
    if x is not q and (x.dtype != dtype or x.device != device or d != q.shape[3] or N != q.shape[0]):
        raise ValueError("%s must share its type, device, rows and head dim with the queries" % what)
    if y is None:
        y_tok = H * d
        y_row = L * y_tok
    else:
        y_shape, y_row, y_tok = _layout(y, "output or gradient")
        if y_shape != shape or y.dtype != dtype or y.device != device:
            raise ValueError("outputs and gradients must share shape, type and device with their heads")
    ps = None if pos is None else pos.shape
    if ps is None or pos.dtype != torch.int32 or ps[-1:] != (L,) or len(ps) > 2 or (len(ps) == 2 and ps[0] != N and ps[0] != 1) \
            or (L > 1 and pos.stride(-1) != 1) or pos.device != device:
        raise ValueError("pos_%s must be int32 [%d, %d], [1, %d] or [%d] with contiguous rows, on the device of q"
                         % (what, N, L, L, L))
    if w is not None:
        _check_weight(w, d, q)
    return H, L, (pos.stride(0) if len(ps) == 2 and ps[0] > 1 else 0), x_row, x_tok, y_row, y_tok


def _check_weight(w: torch.Tensor, d: int, like: torch.Tensor):
    if w.dtype != torch.float32 or w.shape != (d,) or not w.is_contiguous() or w.device != like.device:
        raise ValueError("weights and their gradients must be contiguous float32 [%d] tensors on the queries' device" % d)


_NONE = (0, 0, 0, 0, 0, 0, 0)


def _dims(x, y, pos, steps, weights, interleaved, norm, eps, amplitude):
    """Checks; dims for the sets x (of dx, too) and y (of dy, too)."""
    q, k = x
    dtype, device = q.dtype, q.device
    if dtype not in _DTYPES:
        raise ValueError("q must be float32 or bfloat16")
    a = _set(q, y[0], pos[0], weights[0], q, "q")
    if k is not None:
        b = _set(k, y[1], pos[1], weights[1], q, "k")
    elif pos[1] is not None or weights[1] is not None:
        raise ValueError("pos_k and a weight for keys go with keys")
    else:
        b = _NONE
    if device.type != "cuda" or device.index != torch._C._cuda_getDevice():
        raise ValueError("tensors must be on the current CUDA device")
    st = steps.shape
    if steps.dtype != torch.int64 or len(st) != 1 or not steps.is_contiguous() or steps.device != device:
        raise ValueError("steps must be a contiguous int64 [rot / 2] tensor on the queries' device")
    N, _, _, d = q.shape
    if 2 * st[0] > d:
        raise ValueError("steps are for %d channels, a head has %d" % (2 * st[0], d))
    if not norm and (weights[0] is not None or weights[1] is not None):
        raise ValueError("weights go with norm=True")
    return evo_rope_dims(_DTYPES[dtype], d, 2 * st[0], (_INTERLEAVED if interleaved else 0) | (_NORM if norm else 0),
                         a[0], b[0], eps, amplitude, N, a[1], b[1], a[2], b[2], a[3], b[3], a[4], b[4], a[5], b[5], a[6],
                         b[6])


def _packed(x: torch.Tensor, like: torch.Tensor, stream):
    """A contiguous tensor shaped like x."""
    if stream is None and x.is_contiguous():
        return torch.empty_like(x)
    return _empty(x.shape, x.dtype, like, stream)


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
        out_q = _packed(q, q, stream)
    if k is not None and out_k is None:
        out_k = _packed(k, q, stream)
    st = lib.evo_rope_fwd(dm, q.data_ptr(), _addr(k), _addr(pos_q), _addr(pos_k), steps.data_ptr(), _addr(weight_q),
                          _addr(weight_k), out_q.data_ptr(), _addr(out_k), _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_rope_fwd")
    return out_q, out_k


def rope_bwd_workspace_size(q: torch.Tensor, steps: torch.Tensor, *, k: Optional[torch.Tensor] = None,
                            norm: bool = False) -> int:
    """Bytes of workspace that rope_bwd needs for heads shaped like q and k."""
    N, _, _, d = _layout(q, "q")[0]
    sets = [(0, 0) if x is None else (_layout(x, "heads")[0][2], x.shape[1]) for x in (q, k)]
    heads, lens = zip(*sets)
    tok = tuple(h * d for h in heads)
    row = tuple(l * t for l, t in zip(lens, tok))
    dm = evo_rope_dims(_DTYPES[q.dtype], d, 2 * steps.numel(), _NORM if norm else 0, *heads, 0.0, 1.0, N, *lens, 0, 0, *row,
                       *tok, *row, *tok)
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
            _check_weight(dws[i], w.shape[0], dq)
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
