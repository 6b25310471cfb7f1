"""Host-side checks of the attention to states of another length (no GPU):
exports, every invalid call rejected before any HIP call (fake addresses never
touched), workspace sizes and the binding's refusals."""
import ctypes
import os
import re

import pytest
import torch

from paper_2404_11068_amd import cross
from paper_2404_11068_amd import evo_attn as ea

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, BIG = 0x7f0000000000, 0x10000000
P = lambda x: None if x is None else ctypes.c_void_p(x)
A = lambda i: FAKE + i * BIG


def _lib():
    if not os.path.exists(ea.LIB_PATH):
        pytest.skip("libevoattn.so not built")
    return cross._lib()


def _dims(**kw):
    d = dict(dtype=1, n_heads=8, n_kv_heads=2, head_dim=64, n_rows=4, len_q=10, len_k=300, rows_per_bias=2, q_stride_row=5120,
             q_stride_tok=512, k_stride_row=38400, k_stride_tok=128, o_stride_row=5120, o_stride_tok=512)
    d.update(kw)
    return cross.evo_cross_dims(*d.values())


FWD = dict(q=A(1), k=A(2), v=A(3), gate=A(4), bias=A(5), mask=A(6), out=A(7), lse=A(8), ws=A(9))
BWD = dict(q=A(1), k=A(2), v=A(3), gate=A(4), bias=A(5), mask=A(6), out=A(7), lse=A(8), dout=A(10), dq=A(11), dk=A(12),
           dv=A(13), dgate=A(14), dbias=A(15), ws=A(9))


def _fwd(d, ws_bytes=1 << 40, **kw):
    a = dict(FWD, **kw)
    return _lib().evo_cross_fwd(ctypes.byref(d) if d is not None else None, *[P(x) for x in a.values()], ws_bytes, None)


def _bwd(d, ws_bytes=1 << 40, **kw):
    a = dict(BWD, **kw)
    return _lib().evo_cross_bwd(ctypes.byref(d) if d is not None else None, *[P(x) for x in a.values()], ws_bytes, None)


def test_exports_declared_symbols():
    text = open(os.path.join(ROOT, "include", "evo_cross_attn.h")).read()
    names = re.findall(r"^\s*(?:int|size_t)\s*(evo_\w+)\s*\(", text, flags=re.M)
    assert len(names) == 4
    for n in names:
        assert hasattr(_lib(), n), n


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(n_heads=0), 1), (dict(n_kv_heads=0), 1), (dict(n_kv_heads=3), 1), (dict(n_heads=65536), 2),
    (dict(head_dim=0), 1), (dict(head_dim=12), 2), (dict(head_dim=136), 2), (dict(n_rows=-1), 1), (dict(len_q=-1), 1),
    (dict(len_k=-1), 1), (dict(len_q=1 << 30), 2), (dict(len_k=1 << 31), 2), (dict(n_rows=1 << 41), 2),
    (dict(n_rows=1 << 30, len_k=1, rows_per_bias=1), 2), (dict(rows_per_bias=3), 1), (dict(rows_per_bias=0), 1),
    (dict(q_stride_tok=-512), 1), (dict(q_stride_tok=516), 3), (dict(k_stride_row=38404), 3), (dict(o_stride_row=1 << 41), 2),
    (dict(len_q=1 << 20, len_k=1 << 20), 2),
])
def test_rejects_bad_dims(kw, status):
    assert _fwd(_dims(**kw)) == status and _bwd(_dims(**kw)) == status


def test_outputs_must_not_overlap_themselves():
    assert _fwd(_dims(o_stride_row=0)) == 1 and _fwd(_dims(o_stride_tok=256)) == 1
    assert _bwd(_dims(q_stride_row=0)) == 1 and _bwd(_dims(k_stride_row=0)) == 1 and _bwd(_dims(k_stride_tok=0)) == 1


def test_rejects_bad_pointers():
    d = _dims()
    assert _fwd(None) == 1 and _bwd(None) == 1
    for k in ("q", "k", "v", "out", "lse"):
        assert _fwd(d, **{k: None}) == 1, k
    for k in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "dgate", "dbias", "gate", "bias"):
        assert _bwd(d, **{k: None}) == 1, k
    for k in ("q", "k", "v", "gate", "out"):
        assert _fwd(d, **{k: A(20) + 8}) == 3, k
    assert _fwd(d, bias=A(20) + 1) == 3 and _fwd(d, lse=A(20) + 2) == 3 and _fwd(_dims(dtype=0, q_stride_tok=512), bias=A(20) + 2) == 3
    for k in ("q", "k", "v", "gate", "out", "dout", "dq", "dk", "dv", "dgate"):
        assert _bwd(d, **{k: A(20) + 8}) == 3, k
    for k in ("q", "gate"):
        assert _fwd(d, out=FWD[k]) == 1, k
    assert _fwd(d, out=A(2) + 16) == 1 and _fwd(d, out=A(3) - 512) == 1
    for k in ("q", "gate", "k", "out", "dout"):
        assert _bwd(d, dq=BWD[k]) == 1, k
    for k in ("dq", "dk", "dv", "bias", "v"):
        assert _bwd(d, dgate=BWD[k]) == 1, k
    assert _bwd(d, dv=A(12)) == 1 and _bwd(d, dbias=A(5)) == 1


def test_workspaces():
    # one token of four rows and two key heads, many keys: the keys are split
    lib, d = _lib(), _dims(len_q=1, len_k=3000, q_stride_row=512, k_stride_row=384000, o_stride_row=512)
    need = lib.evo_cross_fwd_workspace_size(ctypes.byref(d))
    assert need > 0
    assert _fwd(d, ws=None) == 4 and _fwd(d, ws_bytes=need - 1) == 4 and _fwd(d, ws=A(9) + 128) == 3
    need = lib.evo_cross_bwd_workspace_size(ctypes.byref(d), 1, 1)
    assert need > 0 and lib.evo_cross_bwd_workspace_size(ctypes.byref(d), 0, 0) > 0
    assert _bwd(d, ws=None) == 4 and _bwd(d, ws_bytes=need - 1) == 4 and _bwd(d, ws=A(9) + 128) == 3
    many = _dims(n_rows=4096, len_k=64, rows_per_bias=4096)
    assert lib.evo_cross_fwd_workspace_size(ctypes.byref(many)) == 0
    assert lib.evo_cross_fwd_workspace_size(ctypes.byref(_dims(dtype=7))) == 0
    # sizes stay sizes for long inputs
    big = _dims(n_rows=1, n_heads=1, n_kv_heads=1, len_q=1, len_k=1 << 24, rows_per_bias=1)
    assert 0 < lib.evo_cross_fwd_workspace_size(ctypes.byref(big)) < 1 << 24


def test_empty_needs_no_pointers():
    none = {k: None for k in FWD}
    assert _fwd(_dims(n_rows=0), **none) == 0 and _fwd(_dims(len_q=0), **none) == 0
    none = {k: None for k in BWD}
    assert _bwd(_dims(n_rows=0), **none) == 0 and _bwd(_dims(len_q=0, len_k=0), **none) == 0


def test_binding_refuses_before_any_launch():
    q, k = torch.zeros(2, 3, 4, 16), torch.zeros(2, 5, 2, 16)
    for kw, what in [(dict(q=q[0]), "N, L, H, d"), (dict(q=q.double()), "float32"), (dict(k=k[:1]), "share"),
                     (dict(k=k.bfloat16()), "share"), (dict(k=torch.zeros(2, 5, 3, 16), v=torch.zeros(2, 5, 3, 16)), "divide"),
                     (dict(q=torch.zeros(2, 3, 4, 32)[..., ::2]), "contiguous"), (dict(), "CUDA")]:
        a = dict(q=q, k=k, v=k)
        a.update(kw)
        with pytest.raises(ValueError, match=what):
            cross.cross_attn_fwd(**a)


@pytest.mark.parametrize("len_q,len_k,most", [(1, 1, 1 << 24), (1, 129, 1 << 23), (129, 1, 1 << 23)])
def test_launches_count_their_threads_in_32_bits(len_q, len_k, most):
    # 2^24 workgroups of 256 threads are one too many; a workspace that is missing shows that a call goes on
    far = {n: FAKE + (i << 38) for i, n in enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv", "lse"))}
    for rows, status in ((most - 1, 4), (most, 2)):
        d = _dims(n_heads=1, n_kv_heads=1, head_dim=8, n_rows=rows, len_q=len_q, len_k=len_k, q_stride_row=8 * len_q,
                  q_stride_tok=8, k_stride_row=8 * len_k, k_stride_tok=8, o_stride_row=8 * len_q, o_stride_tok=8)
        assert _bwd(d, gate=None, bias=None, mask=None, dgate=None, dbias=None, ws=None, **far) == status


def test_a_bias_of_too_many_tiles():
    d = _dims(n_heads=1, n_kv_heads=1, head_dim=8, n_rows=1, len_q=1 << 18, len_k=1 << 18, rows_per_bias=1)
    assert _fwd(d) == 2 and _bwd(d) == 2
