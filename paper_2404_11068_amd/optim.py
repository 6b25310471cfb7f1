"""Python binding of the C ABI in include/evo_optim.h and include/evo_muon.h
(argument marshalling only).

`FusedAdamSWA` packs the pointers of every parameter, gradient and optimizer
state tensor into a device table once (and the chunk list that splits them
into EVO_MT_CHUNK-element work items), then each `step` enqueues the
gradient-norm clipping kernels and the fused Adam + SWA kernel of
``libevoattn.so``.  The table holds raw pointers: rebuild the object if any
of the tensors is reallocated.  No fallback exists.

`FusedMuonSWA` does the same for matrices whose update is orthogonalised by
Newton-Schulz steps; `orthogonalize` is that operation alone, on one matrix or
a stack of them.
"""
from __future__ import annotations

import ctypes
import math
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch

from .evo_attn import EvoAttnError, _empty, _stream, load_library

EVO_MT_CHUNK = 4096


class evo_mt_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("swa", ctypes.c_void_p), ("numel", ctypes.c_int64)]


class evo_mt_chunk(ctypes.Structure):
    _fields_ = [("tensor", ctypes.c_int32), ("index", ctypes.c_int32)]


class evo_adam_swa_hparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("swa_decay", ctypes.c_double),
                ("step", ctypes.c_int64)]


_bound = False


def _lib():
    global _bound
    lib = load_library()
    if not _bound:
        P = ctypes.c_void_p
        lib.evo_mt_chunk_count.argtypes = [ctypes.POINTER(ctypes.c_int64), ctypes.c_int32]
        lib.evo_mt_chunk_count.restype = ctypes.c_int64
        lib.evo_mt_build_chunks.argtypes = [ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, P, ctypes.c_int64]
        lib.evo_mt_build_chunks.restype = ctypes.c_int64
        lib.evo_grad_clip_scale.argtypes = [P, ctypes.c_int32, P, ctypes.c_int32, ctypes.c_float, P, P, P, P]
        lib.evo_grad_clip_scale.restype = ctypes.c_int
        lib.evo_adam_swa_step.argtypes = [ctypes.POINTER(evo_adam_swa_hparams), P, ctypes.c_int32, P, ctypes.c_int32,
                                          P, P]
        lib.evo_adam_swa_step.restype = ctypes.c_int
        _bound = True
    return lib


def _check(t: torch.Tensor, name: str, n: int):
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
        raise ValueError("%s must be a contiguous float32 CUDA tensor of %d elements" % (name, n))


class FusedAdamSWA:
    """Adam + SWA over packed tensors, with optional gradient-norm clipping."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 exp_avg: Optional[Sequence[torch.Tensor]] = None, exp_avg_sq: Optional[Sequence[torch.Tensor]] = None,
                 swa: Optional[Sequence[torch.Tensor]] = None, *, lr=1e-3, betas=(0.9, 0.999), eps=1e-6,
                 weight_decay=0.0, swa_decay=0.999):
        lib = _lib()
        self.params = list(params)
        self.grads = list(grads)
        n = len(self.params)
        if len(self.grads) != n:
            raise ValueError("one gradient per parameter")
        self.exp_avg = list(exp_avg) if exp_avg is not None else [torch.zeros_like(p) for p in self.params]
        self.exp_avg_sq = list(exp_avg_sq) if exp_avg_sq is not None else [torch.zeros_like(p) for p in self.params]
        self.swa = list(swa) if swa is not None else [p.detach().clone() for p in self.params]
        numels = np.array([p.numel() for p in self.params], dtype=np.int64)
        for i in range(n):
            for t, nm in ((self.params[i], "param"), (self.grads[i], "grad"), (self.exp_avg[i], "exp_avg"),
                          (self.exp_avg_sq[i], "exp_avg_sq"), (self.swa[i], "swa")):
                _check(t, "%s[%d]" % (nm, i), int(numels[i]))
        tab = (evo_mt_tensor * max(n, 1))()
        for i in range(n):
            tab[i] = evo_mt_tensor(self.params[i].data_ptr(), self.grads[i].data_ptr(), self.exp_avg[i].data_ptr(),
                                   self.exp_avg_sq[i].data_ptr(), self.swa[i].data_ptr(), int(numels[i]))
        nptr = numels.ctypes.data_as(ctypes.POINTER(ctypes.c_int64))
        nch = int(lib.evo_mt_chunk_count(nptr, n))
        if nch < 0:
            raise ValueError("tensor sizes too large for the chunk table")
        ch = (evo_mt_chunk * max(nch, 1))()
        if int(lib.evo_mt_build_chunks(nptr, n, ch, nch)) != nch:
            raise RuntimeError("evo_mt_build_chunks failed")
        dev = self.params[0].device if n else torch.device("cuda")
        self.tensor_table = torch.frombuffer(bytearray(bytes(tab)), dtype=torch.uint8).to(dev)
        self.chunk_table = torch.frombuffer(bytearray(bytes(ch)), dtype=torch.uint8).to(dev)
        self.n_tensors, self.n_chunks = n, nch
        self.workspace = torch.empty(max(nch, 1), dtype=torch.float32, device=dev)
        self.norm = torch.zeros(1, dtype=torch.float32, device=dev)
        self.scale = torch.ones(1, dtype=torch.float32, device=dev)
        self.lr, self.betas, self.eps, self.weight_decay, self.swa_decay = lr, betas, eps, weight_decay, swa_decay
        self.step_count = 0

    def clip(self, max_norm: float, stream=None):
        """Gradient norm and clipping scale into self.norm / self.scale (device)."""
        st = _lib().evo_grad_clip_scale(self.tensor_table.data_ptr(), self.n_tensors, self.chunk_table.data_ptr(),
                                        self.n_chunks, float(max_norm), self.workspace.data_ptr(),
                                        self.norm.data_ptr(), self.scale.data_ptr(), _stream(stream))
        if st:
            raise EvoAttnError(st, "evo_grad_clip_scale")

    def step(self, max_norm: Optional[float] = None, stream=None, step: Optional[int] = None):
        """One optimizer step (clipping first when max_norm is given)."""
        if max_norm is not None:
            self.clip(max_norm, stream)
        self.step_count = self.step_count + 1 if step is None else step
        hp = evo_adam_swa_hparams(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                                  self.swa_decay, self.step_count)
        st = _lib().evo_adam_swa_step(ctypes.byref(hp), self.tensor_table.data_ptr(), self.n_tensors,
                                      self.chunk_table.data_ptr(), self.n_chunks,
                                      self.scale.data_ptr() if max_norm is not None else None, _stream(stream))
        if st:
            raise EvoAttnError(st, "evo_adam_swa_step")


# ---------------------------------------------------------------------------
# Orthogonalised updates (include/evo_muon.h)

#: quintic Newton-Schulz coefficients: the steepest slope at zero that still
#: keeps the singular values within about 0.7 .. 1.2
NEWTON_SCHULZ_COEFS = (3.4445, -4.7750, 2.0315)

_ORTH_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class evo_orth_dims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("steps", ctypes.c_int32), ("n_batch", ctypes.c_int64),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("a", ctypes.c_double), ("b", ctypes.c_double),
                ("c", ctypes.c_double), ("eps", ctypes.c_double), ("reserved", ctypes.c_int64)]


class evo_muon_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("momentum", ctypes.c_void_p),
                ("swa", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("update_scale", ctypes.c_double)]


class evo_muon_hparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("swa_decay", ctypes.c_double), ("a", ctypes.c_double), ("b", ctypes.c_double),
                ("c", ctypes.c_double), ("eps", ctypes.c_double), ("steps", ctypes.c_int32),
                ("nesterov", ctypes.c_int32)]


_muon_bound = False


def _muon_lib():
    global _muon_bound
    lib = load_library()
    if not _muon_bound:
        P = ctypes.c_void_p
        lib.evo_orthogonalize_workspace_size.argtypes = [ctypes.POINTER(evo_orth_dims)]
        lib.evo_orthogonalize_workspace_size.restype = ctypes.c_size_t
        lib.evo_orthogonalize.argtypes = [ctypes.POINTER(evo_orth_dims), P, P, P, ctypes.c_size_t, P]
        lib.evo_orthogonalize.restype = ctypes.c_int
        lib.evo_muon_plan_bytes.argtypes = [P, ctypes.c_int32]
        lib.evo_muon_plan_bytes.restype = ctypes.c_int64
        lib.evo_muon_build_plan.argtypes = [P, ctypes.c_int32, P, ctypes.c_size_t]
        lib.evo_muon_build_plan.restype = ctypes.c_int
        lib.evo_muon_workspace_size.argtypes = [P]
        lib.evo_muon_workspace_size.restype = ctypes.c_size_t
        lib.evo_muon_step.argtypes = [ctypes.POINTER(evo_muon_hparams), P, P, P, P, ctypes.c_size_t, P]
        lib.evo_muon_step.restype = ctypes.c_int
        _muon_bound = True
    return lib


def _orth_dims(shape, dtype, steps, coefs, eps) -> evo_orth_dims:
    if len(shape) not in (2, 3) or dtype not in _ORTH_DTYPES:
        raise ValueError("x must be a float32 or bfloat16 matrix [m, n] or stack of matrices [N, m, n]")
    n = shape[0] if len(shape) == 3 else 1
    a, b, c = coefs
    return evo_orth_dims(_ORTH_DTYPES[dtype], steps, n, shape[-2], shape[-1], a, b, c, eps, 0)


def orthogonalize_workspace_size(shape, dtype, *, steps: int = 5, coefs: Tuple[float, float, float] = NEWTON_SCHULZ_COEFS,
                                 eps: float = 1e-7) -> int:
    d = _orth_dims(tuple(shape), dtype, steps, coefs, eps)
    return int(_muon_lib().evo_orthogonalize_workspace_size(ctypes.byref(d)))


def orthogonalize(x: torch.Tensor, *, steps: int = 5, coefs: Tuple[float, float, float] = NEWTON_SCHULZ_COEFS,
                  eps: float = 1e-7, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """The matrix x [m, n], or every matrix of a stack [N, m, n], with its
    singular values brought near one by `steps` Newton-Schulz steps
    X <- a X + (b A + c A^2) X, A = X X^T, from X = x / max(|x|_F, eps).
    fp32 to fp32's precision; bf16 as the fp32 result rounded once.  out may be x."""
    lib = _muon_lib()
    d = _orth_dims(x.shape, x.dtype, steps, coefs, eps)
    if not x.is_contiguous() or not x.is_cuda or x.get_device() != torch._C._cuda_getDevice():
        raise ValueError("x must be contiguous and on the current CUDA device")
    if out is None:
        out = _empty(x.shape, x.dtype, x, stream)
    elif out.shape != x.shape or out.dtype != x.dtype or not out.is_contiguous() or out.device != x.device:
        raise ValueError("out must be a contiguous tensor like x")
    if workspace is None:
        ws_bytes = lib.evo_orthogonalize_workspace_size(d)
        workspace = _empty((max(ws_bytes, 1),), torch.uint8, x, stream)
    elif not workspace.is_contiguous() or workspace.device != x.device:
        raise ValueError("workspace must be contiguous and on the device of x")
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    st = lib.evo_orthogonalize(d, x.data_ptr(), out.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(stream))
    if st:
        raise EvoAttnError(st, "evo_orthogonalize")
    return out


class FusedMuonSWA:
    """Muon + SWA over matrices: momentum, the orthogonalised update, weight
    decay and the weight average.  Vectors (biases, LayerNorm parameters) and
    embeddings belong to FusedAdamSWA, whose `scale` (after `clip`) can be
    passed to `step` so that both clip by the same norm.

    Stacked projections are given as their matrices, e.g. the q, k, v and
    gate rows of one weight as `list(w.view(4, -1, w.shape[1]))`.

    Construction checks every tensor and builds the plan on the host, once: 9 ms
    for the 2263 matrices of an AlphaFold-sized model, four of its steps.

    adjust: factor of the update of an m x n matrix: "spectral" gives
    sqrt(max(1, m / n)), "rms" 0.2 sqrt(max(m, n)) (entries about as large as
    Adam's), "none" 1."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 momentum: Optional[Sequence[torch.Tensor]] = None, swa: Optional[Sequence[torch.Tensor]] = None, *,
                 lr=0.02, momentum_decay=0.95, nesterov=True, weight_decay=0.0, swa_decay=0.999, steps=5,
                 coefs=NEWTON_SCHULZ_COEFS, eps=1e-7, adjust="spectral"):
        lib = _muon_lib()
        self.params, self.grads = list(params), list(grads)
        n = len(self.params)
        if adjust not in ("spectral", "rms", "none"):
            raise ValueError("adjust must be 'spectral', 'rms' or 'none'")
        if len(self.grads) != n:
            raise ValueError("one gradient per parameter")
        for i, p in enumerate(self.params):
            if p.dim() != 2:
                raise ValueError("param[%d] must be a matrix: vectors go to FusedAdamSWA" % i)
        self.momentum = list(momentum) if momentum is not None else [torch.zeros_like(p) for p in self.params]
        self.swa = list(swa) if swa is not None else [p.detach().clone() for p in self.params]
        if len(self.momentum) != n or len(self.swa) != n:
            raise ValueError("one momentum and one swa tensor per parameter")
        dev = self.params[0].device if n else torch.device("cuda", torch.cuda.current_device())
        tab = np.zeros(n, dtype=np.dtype(evo_muon_tensor))
        for i, p in enumerate(self.params):
            for t, nm in ((p, "param"), (self.grads[i], "grad"), (self.momentum[i], "momentum"), (self.swa[i], "swa")):
                if t.dtype != torch.float32 or t.shape != p.shape or not t.is_cuda or t.device != dev \
                        or not t.is_contiguous():
                    raise ValueError("%s[%d] must be a contiguous float32 CUDA matrix like its parameter" % (nm, i))
            r, c = p.shape
            f = 1.0 if adjust == "none" or r * c == 0 else \
                math.sqrt(max(1.0, r / c)) if adjust == "spectral" else 0.2 * math.sqrt(max(r, c))
            tab[i] = (p.data_ptr(), self.grads[i].data_ptr(), self.momentum[i].data_ptr(), self.swa[i].data_ptr(),
                      r, c, f)
        # all matrices are worked on at the same time: what one writes, no other may read or write
        ends = []
        for kind, ts in ((1, self.params), (1, self.momentum), (1, self.swa), (0, self.grads)):
            ends += [(t.data_ptr(), t.data_ptr() + 4 * t.numel(), kind) for t in ts if t.numel()]
        ends.sort()
        written = read = 0
        for begin, end, kind in ends:
            if begin < written or (kind and begin < read):
                raise ValueError("parameters, momenta and averages must not overlap each other or a gradient")
            written, read = (max(written, end), read) if kind else (written, max(read, end))
        size = int(lib.evo_muon_plan_bytes(tab.ctypes.data, n))
        if size < 0:
            raise ValueError("a matrix is too large for the plan")
        self.plan = np.zeros((size + 7) // 8, dtype=np.int64)  # host copy
        st = lib.evo_muon_build_plan(tab.ctypes.data, n, self.plan.ctypes.data, size)
        if st:
            raise EvoAttnError(st, "evo_muon_build_plan")
        self.device = dev
        self.plan_device = torch.from_numpy(self.plan).to(dev)
        self.workspace = torch.empty(max(int(lib.evo_muon_workspace_size(self.plan.ctypes.data)), 1),
                                     dtype=torch.uint8, device=dev)
        self.lr, self.momentum_decay, self.nesterov = lr, momentum_decay, nesterov
        self.weight_decay, self.swa_decay = weight_decay, swa_decay
        self.steps, self.coefs, self.eps = steps, coefs, eps

    def step(self, grad_scale: Optional[torch.Tensor] = None, stream=None):
        """One step; grad_scale: a device float32 scalar that multiplies every
        gradient (FusedAdamSWA.scale).  Steps of one object share its
        workspace: they must not overlap in time."""
        if self.device.index != torch.cuda.current_device():
            raise ValueError("the tensors are not on the current CUDA device")
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                       or grad_scale.device != self.device):
            raise ValueError("grad_scale must be one float32 on the tensors' device")
        hp = evo_muon_hparams(self.lr, self.momentum_decay, self.weight_decay, self.swa_decay, *self.coefs, self.eps,
                              self.steps, int(self.nesterov))
        st = _muon_lib().evo_muon_step(ctypes.byref(hp), self.plan.ctypes.data, self.plan_device.data_ptr(),
                                       grad_scale.data_ptr() if grad_scale is not None else None,
                                       self.workspace.data_ptr(), self.workspace.numel(), _stream(stream))
        if st:
            raise EvoAttnError(st, "evo_muon_step")
