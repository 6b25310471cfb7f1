"""Python binding of the C ABI in include/evo_cross_attn.h (argument marshalling only).

The gated attention of queries to states of another length runs in
``libevoattn.so``; this module passes torch tensors' device pointers and raises
on a nonzero status.  No fallback exists.

  q, gate, dq, dgate : [N, Lq, H, d]; k, v, dk, dv : [N, Lk, Hk, d]; out, dout : [N, Lq, H, d], bf16 or fp32,
      the [H, d] block of each token contiguous; within each of the three groups one (row, token) stride pair.
      Any lengths; Hk divides H, query head i reads key head i // (H // Hk).  Inputs may repeat rows (expand).
  bias, dbias : [B, H, Lq, Lk] contiguous, of the queries' type, B = N // rows_per_bias
  key_mask : [N, Lk] uint8 or bool (nonzero = keep)
  lse : [N, H, Lq] float32
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from .evo_attn import EvoAttnError, _DTYPES, _empty, _stream, load_library


class evo_cross_dims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)] + [(n, ctypes.c_int64) for n in (
                    "n_rows", "len_q", "len_k", "rows_per_bias", "q_stride_row", "q_stride_tok", "k_stride_row",
                    "k_stride_tok", "o_stride_row", "o_stride_tok")]


_bound = False


def _lib():
    global _bound
    lib = load_library()
    if not _bound:
        P = ctypes.c_void_p
        D = ctypes.POINTER(evo_cross_dims)
        lib.evo_cross_fwd_workspace_size.argtypes = [D]
        lib.evo_cross_fwd_workspace_size.restype = ctypes.c_size_t
        lib.evo_cross_fwd.argtypes = [D] + [P] * 9 + [ctypes.c_size_t, P]
        lib.evo_cross_fwd.restype = ctypes.c_int
        lib.evo_cross_bwd_workspace_size.argtypes = [D, ctypes.c_int, ctypes.c_int]
        lib.evo_cross_bwd_workspace_size.restype = ctypes.c_size_t
        lib.evo_cross_bwd.argtypes = [D] + [P] * 15 + [ctypes.c_size_t, P]
        lib.evo_cross_bwd.restype = ctypes.c_int
        _bound = True
    return lib


def _block(x: torch.Tensor, what: str):
    """(shape, (row, token) strides) of a token tensor; an axis of one entry, whose stride says nothing, counts as packed."""
    shape = x.shape
    if len(shape) != 4:
        raise ValueError("%s must be [N, L, H, d]" % what)
    N, L, H, d = shape
    sr, st, sh, sd = x.stride()
    if (d > 1 and sd != 1) or (H > 1 and sh != d):
        raise ValueError("the [H, d] block of each token of %s must be contiguous" % what)
    if L <= 1:
        st = H * d
    return shape, (sr if N > 1 and L > 0 else L * st, st)


def _like(x: Optional[torch.Tensor], ref: torch.Tensor, strides, what: str):
    if x is None:
        return
    if x.shape != ref.shape or x.dtype != ref.dtype or x.device != ref.device or _block(x, what)[1] != strides:
        raise ValueError("%s must share shape, strides, type and device with its group" % what)


def _dims(q, k, v, gate, bias, key_mask, rows_per_bias):
    """Checks of the inputs; the dims without the o strides, and the q and k strides."""
    (N, Lq, H, d), qs = _block(q, "q")
    (Nk, Lk, Hk, dk), ks = _block(k, "k")
    if q.dtype not in _DTYPES:
        raise ValueError("dtype must be float32 or bfloat16")
    if Nk != N or dk != d or k.dtype != q.dtype or k.device != q.device:
        raise ValueError("k must share its type, device, rows and head dim with q")
    if Hk < 1 or H % Hk:
        raise ValueError("the number of key heads must divide that of query heads")
    if q.device.type != "cuda" or q.device.index != torch._C._cuda_getDevice():
        raise ValueError("tensors must be on the current CUDA device")
    _like(v, k, ks, "v")
    _like(gate, q, qs, "gate")
    rpb = max(N, 1) if rows_per_bias is None else rows_per_bias
    if rpb < 1 or N % rpb:
        raise ValueError("rows_per_bias must divide the rows")
    if bias is not None and (bias.shape != (N // rpb, H, Lq, Lk) or bias.dtype != q.dtype or not bias.is_contiguous()
                             or bias.device != q.device):
        raise ValueError("bias must be a contiguous %s tensor of shape %s" % (q.dtype, (N // rpb, H, Lq, Lk)))
    if key_mask is not None and (key_mask.shape != (N, Lk) or key_mask.dtype not in (torch.uint8, torch.bool)
                                 or not key_mask.is_contiguous() or key_mask.device != q.device):
        raise ValueError("key_mask must be a contiguous uint8 or bool tensor of shape %s" % ((N, Lk),))
    return evo_cross_dims(_DTYPES[q.dtype], H, Hk, d, N, Lq, Lk, rpb, qs[0], qs[1], ks[0], ks[1], Lq * H * d, H * d), qs, ks


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _workspace(ws, need: int, like: torch.Tensor, stream):
    if ws is None:
        return (_empty((need,), torch.uint8, like, stream) if need else None), need
    if ws.device != like.device or not ws.is_contiguous():
        raise ValueError("workspace must be contiguous and on the device of q")
    return ws, ws.numel() * ws.element_size()


def _lse(lse, q):
    N, Lq, H, _ = q.shape
    if lse.shape != (N, H, Lq) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != q.device:
        raise ValueError("lse must be a contiguous float32 tensor of shape %s" % ((N, H, Lq),))


def cross_attn_fwd_workspace_size(q: torch.Tensor, k: torch.Tensor) -> int:
    """Bytes of workspace that cross_attn_fwd needs for tensors like q and k."""
    return int(_lib().evo_cross_fwd_workspace_size(_dims(q, k, k, None, None, None, None)[0]))


def cross_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: Optional[torch.Tensor] = None,
                   bias: Optional[torch.Tensor] = None, key_mask: Optional[torch.Tensor] = None, *, rows_per_bias=None,
                   out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """sigmoid(gate) * softmax(q k^T / sqrt(d) + bias) v over the kept keys; returns (out, lse).  See
    include/evo_cross_attn.h."""
    lib = _lib()
    dm, _, _ = _dims(q, k, v, gate, bias, key_mask, rows_per_bias)
    if out is None:
        out = torch.empty_like(q) if stream is None and q.is_contiguous() else _empty(q.shape, q.dtype, q, stream)
    else:
        os_ = _block(out, "out")[1]
        _like(out, q, os_, "out")
        dm.o_stride_row, dm.o_stride_tok = os_
    if lse is None:
        lse = _empty((dm.n_rows, dm.n_heads, dm.len_q), torch.float32, q, stream)
    else:
        _lse(lse, q)
    workspace, nbytes = _workspace(workspace, lib.evo_cross_fwd_workspace_size(dm), q, stream)
    st = lib.evo_cross_fwd(dm, q.data_ptr(), k.data_ptr(), v.data_ptr(), _addr(gate), _addr(bias), _addr(key_mask),
                           out.data_ptr(), lse.data_ptr(), _addr(workspace), nbytes, _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_cross_fwd")
    return out, lse


def cross_attn_bwd_workspace_size(q: torch.Tensor, k: torch.Tensor, has_gate: bool = False, has_bias: bool = False,
                                  rows_per_bias=None) -> int:
    """Bytes of workspace that cross_attn_bwd needs for tensors like q and k."""
    dm = _dims(q, k, k, None, None, None, rows_per_bias)[0]
    return int(_lib().evo_cross_bwd_workspace_size(dm, int(has_gate), int(has_bias)))


def _grad(given, like, strides, what, stream):
    """A gradient laid out like its input (whose layout it shares), or the one given."""
    if given is not None:
        _like(given, like, strides, what)
        return given
    if like.is_contiguous():
        return _empty(like.shape, like.dtype, like, stream)
    if 0 in [s for s, n in zip(like.stride(), like.shape) if n > 1]:
        raise ValueError("the gradient of an input that repeats entries (expand) cannot be laid out like it: "
                         "pass a contiguous input")
    size = sum((n - 1) * s for n, s in zip(like.shape, like.stride())) + 1 if like.numel() else 0
    return _empty((size,), like.dtype, like, stream).as_strided(like.shape, like.stride())


def cross_attn_bwd(q, k, v, gate, bias, key_mask, out, lse, dout, *, rows_per_bias=None, dq=None, dk=None, dv=None,
                   dgate=None, dbias=None, workspace=None, stream=None):
    """Backward pass; returns (dq, dk, dv, dgate or None, dbias or None), dbias in the bias' type."""
    lib = _lib()
    dm, qs, ks = _dims(q, k, v, gate, bias, key_mask, rows_per_bias)
    os_ = _block(out, "out")[1]
    _like(out, q, os_, "out")
    _like(dout, q, os_, "dout")
    dm.o_stride_row, dm.o_stride_tok = os_
    _lse(lse, q)
    if (gate is None and dgate is not None) or (bias is None and dbias is not None):
        raise ValueError("dgate and dbias go with gate and bias")
    dq = _grad(dq, q, qs, "dq", stream)
    dk, dv = _grad(dk, k, ks, "dk", stream), _grad(dv, k, ks, "dv", stream)
    if gate is not None:
        dgate = _grad(dgate, q, qs, "dgate", stream)
    if bias is not None:
        if dbias is None:
            dbias = _empty(bias.shape, bias.dtype, q, stream)
        elif dbias.shape != bias.shape or dbias.dtype != bias.dtype or not dbias.is_contiguous() or dbias.device != q.device:
            raise ValueError("dbias must be contiguous and shaped and typed like the bias")
    need = lib.evo_cross_bwd_workspace_size(dm, int(gate is not None), int(bias is not None))
    workspace, nbytes = _workspace(workspace, need, q, stream)
    st = lib.evo_cross_bwd(dm, q.data_ptr(), k.data_ptr(), v.data_ptr(), _addr(gate), _addr(bias), _addr(key_mask),
                           out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                           _addr(dgate), _addr(dbias), _addr(workspace), nbytes, _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_cross_bwd")
    return dq, dk, dv, dgate, dbias
