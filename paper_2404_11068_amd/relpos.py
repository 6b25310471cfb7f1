"""Python binding of the C ABI in include/evo_relpos.h (argument marshalling only).

The learned relative position bias runs in ``libevoattn.so``; this module
passes torch tensors' device pointers and raises on a nonzero status.  No
fallback exists.

  pos_i, pos_j : int32 [B, Li], [B, Lj] (or [Li], [Lj] for one batch entry): residue or token numbers
  seg_i, seg_j : int32 like them, or None: pairs of different segments (chains) take the last bucket
  edges : int32 [E], ascending: the first difference pos_i - pos_j of every bucket but the lowest
  table : fp32 [H, buckets], buckets = E + 1, and one more with segments
  base, out : [B, H, Li, Lj] bf16 or fp32, the bias layout of evo_attn_fwd
  dbias : fp32 [B, H, Li, Lj], as evo_attn_bwd returns it
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .evo_attn import EVO_DTYPE_F32, EvoAttnError, _DTYPES, _empty, _stream, load_library


class evo_relpos_dims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_edges", ctypes.c_int32),
                ("has_seg", ctypes.c_int32), ("n_batch", ctypes.c_int64), ("len_i", ctypes.c_int64),
                ("len_j", ctypes.c_int64), ("reserved", ctypes.c_int64)]


_bound = False


def _lib():
    global _bound
    lib = load_library()
    if not _bound:
        P = ctypes.c_void_p
        D = ctypes.POINTER(evo_relpos_dims)
        lib.evo_relpos_fwd.argtypes = [D] + [P] * 9
        lib.evo_relpos_fwd.restype = ctypes.c_int
        lib.evo_relpos_bwd_workspace_size.argtypes = [D]
        lib.evo_relpos_bwd_workspace_size.restype = ctypes.c_size_t
        lib.evo_relpos_bwd.argtypes = [D] + [P] * 8 + [ctypes.c_size_t, P]
        lib.evo_relpos_bwd.restype = ctypes.c_int
        _bound = True
    return lib


def relpos_edges_clip(max_offset: int, device="cuda") -> torch.Tensor:
    """Edges of the 2 * max_offset + 1 buckets of differences clipped at +-max_offset
    (AlphaFold's relative positions: 32, which makes 65 buckets)."""
    if max_offset < 0:
        raise ValueError("max_offset must not be negative")
    return torch.arange(1 - max_offset, max_offset + 1, dtype=torch.int32, device=device)


def relpos_edges_log(n_side: int, max_distance: int, device="cuda") -> torch.Tensor:
    """Edges of 2 * n_side - 1 buckets, symmetric around difference 0: single
    distances up to n_side // 2, from there on bucket widths that grow by a
    constant factor; distances of max_distance and more share the last
    bucket of their side (fewer buckets where steps below one would repeat
    an edge)."""
    half = n_side // 2
    if n_side < 3 or max_distance <= half:
        raise ValueError("n_side must be at least 3 and max_distance larger than n_side // 2")
    near = list(range(1, half + 1))
    steps = n_side - 1 - half
    far = [min(max_distance, max(half + 1, math.ceil(half * (max_distance / half) ** (k / steps))))
           for k in range(1, steps)] + [max_distance]
    side = near + sorted(set(far))
    return torch.tensor([1 - e for e in reversed(side)] + side, dtype=torch.int32, device=device)


def _index(pos_i, pos_j, edges, seg_i, seg_j, like: torch.Tensor):
    """Checks of the index tensors; returns (B, Li, Lj, E)."""
    si, sj, se = pos_i.shape, pos_j.shape, edges.shape
    if len(si) not in (1, 2) or len(sj) != len(si) or len(se) != 1:
        raise ValueError("pos_i and pos_j must be [B, Li] and [B, Lj] (or [Li] and [Lj]), edges [E]")
    if len(si) == 2 and si[0] != sj[0]:
        raise ValueError("pos_i and pos_j must have the same batch size")
    ts = (pos_i, pos_j, edges)
    if seg_i is not None or seg_j is not None:
        if seg_i is None or seg_j is None:
            raise ValueError("seg_i and seg_j go together")
        if seg_i.shape != si or seg_j.shape != sj:
            raise ValueError("segments must be shaped like the positions")
        ts = (pos_i, pos_j, edges, seg_i, seg_j)
    dev = like.device
    for t in ts:
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError("positions, segments and edges must be contiguous int32")
        if t.device != dev:
            raise ValueError("tensors must be on one device")
    if dev.type != "cuda" or dev.index != torch._C._cuda_getDevice():
        raise ValueError("tensors must be on the current CUDA device")
    return (si[0] if len(si) == 2 else 1), si[-1], sj[-1], se[0]


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def relpos_bias_fwd(pos_i: torch.Tensor, pos_j: torch.Tensor, edges: torch.Tensor, table: torch.Tensor, *,
                    seg_i: Optional[torch.Tensor] = None, seg_j: Optional[torch.Tensor] = None,
                    base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, dtype=None,
                    stream=None) -> torch.Tensor:
    """Bias [B, H, Li, Lj] for evo_attn_fwd: table[h, bucket(i, j)], added to
    base when given (out=base adds in place).  dtype: of the result; that of
    out or base when one is given, bfloat16 otherwise."""
    lib = _lib()
    B, Li, Lj, E = _index(pos_i, pos_j, edges, seg_i, seg_j, table)
    seg = 0 if seg_i is None else 1
    H = table.shape[0]
    if table.shape != (H, E + 1 + seg) or H < 1 or table.dtype != torch.float32 or not table.is_contiguous():
        raise ValueError("table must be a contiguous float32 [H, %d] tensor" % (E + 1 + seg))
    if dtype is None:
        dtype = out.dtype if out is not None else base.dtype if base is not None else torch.bfloat16
    if dtype not in _DTYPES:
        raise ValueError("dtype must be float32 or bfloat16")
    shape = (B, H, Li, Lj)
    given = (base, out)
    if out is None:
        out = _empty(shape, dtype, table, stream)
    for t in given:
        if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous()
                              or t.device != table.device):
            raise ValueError("base and out must be contiguous %s tensors of shape %s" % (dtype, shape))
    d = evo_relpos_dims(_DTYPES[dtype], H, E, seg, B, Li, Lj, 0)
    st = lib.evo_relpos_fwd(d, pos_i.data_ptr(), pos_j.data_ptr(), _addr(seg_i), _addr(seg_j), edges.data_ptr(),
                            table.data_ptr(), _addr(base), out.data_ptr(), _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_relpos_fwd")
    return out


def relpos_bias_bwd_workspace_size(B: int, H: int, Li: int, Lj: int, n_edges: int, has_seg: bool = False) -> int:
    d = evo_relpos_dims(EVO_DTYPE_F32, H, n_edges, int(has_seg), B, Li, Lj, 0)
    return int(_lib().evo_relpos_bwd_workspace_size(ctypes.byref(d)))


def relpos_bias_bwd(pos_i: torch.Tensor, pos_j: torch.Tensor, edges: torch.Tensor, dbias: torch.Tensor, *,
                    seg_i: Optional[torch.Tensor] = None, seg_j: Optional[torch.Tensor] = None,
                    dtable: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Gradient [H, buckets] (fp32) of relpos_bias_fwd's table for the upstream
    gradient dbias, which is the gradient of its base, too."""
    lib = _lib()
    B, Li, Lj, E = _index(pos_i, pos_j, edges, seg_i, seg_j, dbias)
    H = dbias.shape[1] if dbias.dim() == 4 else 0
    if dbias.shape != (B, H, Li, Lj) or H < 1 or dbias.dtype != torch.float32 or not dbias.is_contiguous():
        raise ValueError("dbias must be a contiguous float32 [%d, H, %d, %d] tensor" % (B, Li, Lj))
    seg = 0 if seg_i is None else 1
    shape = (H, E + 1 + seg)
    if dtable is None:
        dtable = _empty(shape, torch.float32, dbias, stream)
    elif dtable.shape != shape or dtable.dtype != torch.float32 or not dtable.is_contiguous() \
            or dtable.device != dbias.device:
        raise ValueError("dtable must be a contiguous float32 [%d, %d] tensor" % shape)
    d = evo_relpos_dims(EVO_DTYPE_F32, H, E, seg, B, Li, Lj, 0)
    if workspace is None:
        need = ws_bytes = lib.evo_relpos_bwd_workspace_size(d)
        workspace = _empty((need,), torch.uint8, dbias, stream)
    elif workspace.device != dbias.device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on the device of dbias")
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    st = lib.evo_relpos_bwd(d, pos_i.data_ptr(), pos_j.data_ptr(), _addr(seg_i), _addr(seg_j), edges.data_ptr(),
                            dbias.data_ptr(), dtable.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_relpos_bwd")
    return dtable
