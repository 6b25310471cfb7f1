"""Host-side checks of the relative position bias (no GPU): exports, every
invalid call rejected before any HIP call (fake addresses never touched), and
the binding's refusals and edge tables."""
import ctypes
import os
import re

import pytest
import torch

from paper_2404_11068_amd import evo_attn as ea
from paper_2404_11068_amd import relpos as rp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000
P = lambda x: None if x is None else ctypes.c_void_p(x)


def _lib():
    if not os.path.exists(ea.LIB_PATH):
        pytest.skip("libevoattn.so not built")
    return rp._lib()


def _dims(**kw):
    d = dict(dtype=1, n_heads=8, n_edges=64, has_seg=0, n_batch=1, len_i=256, len_j=256, reserved=0)
    d.update(kw)
    return rp.evo_relpos_dims(*d.values())


def _fwd(d, pos_i=FAKE, pos_j=FAKE + 4096, seg_i=None, seg_j=None, edges=FAKE + 8192, table=FAKE + 16384, base=None,
         out=FAKE + 0x1000000):
    return _lib().evo_relpos_fwd(ctypes.byref(d) if d is not None else None, P(pos_i), P(pos_j), P(seg_i), P(seg_j),
                                 P(edges), P(table), P(base), P(out), None)


def _bwd(d, pos_i=FAKE, pos_j=FAKE + 4096, seg_i=None, seg_j=None, edges=FAKE + 8192, dbias=FAKE + 0x1000000,
         dtable=FAKE + 16384, ws=FAKE + 0x8000000, ws_bytes=1 << 40):
    return _lib().evo_relpos_bwd(ctypes.byref(d) if d is not None else None, P(pos_i), P(pos_j), P(seg_i), P(seg_j),
                                 P(edges), P(dbias), P(dtable), P(ws), ws_bytes, None)


def test_exports_declared_symbols():
    text = open(os.path.join(ROOT, "include", "evo_relpos.h")).read()
    for n in re.findall(r"^\s*(?:int|size_t)\s*(evo_\w+)\s*\(", text, flags=re.M):
        assert hasattr(_lib(), n), n


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(n_heads=0), 1), (dict(n_heads=65536), 2), (dict(n_edges=-1), 1),
    (dict(n_edges=1023), 2), (dict(has_seg=2), 1), (dict(n_batch=-1), 1), (dict(len_i=-1), 1), (dict(len_j=-1), 1),
    (dict(len_i=(1 << 20) + 1), 2), (dict(len_i=1 << 20, len_j=1 << 20, n_heads=2), 2),
    (dict(n_batch=1 << 40, n_heads=2, len_i=1, len_j=1), 2), (dict(reserved=1), 1),
])
def test_rejects_bad_dims(kw, status):
    d = _dims(**kw)
    assert _fwd(d) == status and _bwd(d) == status
    assert _lib().evo_relpos_bwd_workspace_size(ctypes.byref(d)) == 0


def test_rejects_bad_pointers():
    d = _dims()
    assert _fwd(None) == 1 and _bwd(None) == 1
    for k in ("pos_i", "pos_j", "edges", "table", "out"):
        assert _fwd(d, **{k: None}) == 1, k
    for k in ("pos_i", "pos_j", "edges", "dbias", "dtable"):
        assert _bwd(d, **{k: None}) == 1, k
    assert _fwd(d, seg_i=FAKE, seg_j=FAKE) == 1                     # segments that the dims do not name
    s = _dims(has_seg=1)
    assert _fwd(s) == 1 and _fwd(s, seg_i=FAKE) == 1 and _bwd(s, seg_j=FAKE) == 1
    for k in ("pos_i", "pos_j", "edges", "table"):
        assert _fwd(d, **{k: FAKE + 2}) == 3, k
    assert _fwd(d, out=FAKE + 0x1000001) == 3 and _fwd(d, base=FAKE + 0x3000001) == 3
    assert _fwd(_dims(dtype=0), out=FAKE + 0x1000002) == 3
    assert _fwd(d, base=FAKE + 0x1000000 + 2) == 1                  # overlaps out
    assert _fwd(d, out=FAKE + 16384) == 1                           # is the table
    assert _bwd(d, dbias=FAKE + 0x1000002) == 3 and _bwd(d, dtable=FAKE + 2) == 3
    need = _lib().evo_relpos_bwd_workspace_size(ctypes.byref(d))
    if need:
        assert _bwd(d, ws=None) == 4 and _bwd(d, ws_bytes=need - 1) == 4 and _bwd(d, ws=FAKE + 8) == 3


def test_empty_forward_needs_no_pointers():
    assert _fwd(_dims(len_i=0), pos_i=None, pos_j=None, edges=None, table=None, out=None) == 0


def test_edge_tables():
    assert rp.relpos_edges_clip(2, device="cpu").tolist() == [-1, 0, 1, 2]
    assert rp.relpos_edges_clip(0, device="cpu").tolist() == []
    assert rp.relpos_edges_clip(32, device="cpu").numel() == 64
    for n, far in ((3, 2), (4, 100), (16, 128), (32, 20), (64, 1024)):
        e = rp.relpos_edges_log(n, far, device="cpu").tolist()
        assert e == sorted(set(e)) and e == [1 - x for x in reversed(e)]
        assert e[-1] == far
        assert len(e) <= 2 * (n - 1) and set(range(1, n // 2 + 1)) <= set(e)
    assert rp.relpos_edges_log(16, 128, device="cpu").numel() == 30
    for bad in ((2, 5), (8, 4)):
        with pytest.raises(ValueError):
            rp.relpos_edges_log(*bad, device="cpu")
    with pytest.raises(ValueError):
        rp.relpos_edges_clip(-1, device="cpu")


def test_binding_refuses_before_any_launch():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    e, t = i(4), torch.zeros(2, 5)
    bad = [
        (dict(pos_i=i(1, 3), pos_j=i(4)), "pos_i"), (dict(pos_i=i(2, 3)), "batch"),
        (dict(seg_i=i(1, 3)), "together"), (dict(seg_i=i(1, 3), seg_j=i(1, 3)), "shaped"),
        (dict(pos_i=i(1, 3).long()), "int32"), (dict(edges=i(4, 1)), "edges"),
        (dict(pos_j=i(1, 8)[:, ::2]), "contiguous"), (dict(), "CUDA"),
    ]
    for kw, what in bad:
        args = dict(pos_i=i(1, 3), pos_j=i(1, 4), edges=e)
        args.update(kw)
        with pytest.raises(ValueError, match=what):
            rp.relpos_bias_fwd(args.pop("pos_i"), args.pop("pos_j"), args.pop("edges"), t, **args)
