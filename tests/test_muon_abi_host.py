"""Host-side checks of the orthogonalised step (no GPU): exports, plans, and
rejection of invalid calls before any HIP call (fake addresses never touched)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2404_11068_amd import evo_attn as ea
from paper_2404_11068_amd import optim as op

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000
BIG = 1 << 50


def _lib():
    if not os.path.exists(ea.LIB_PATH):
        pytest.skip("libevoattn.so not built")
    return op._muon_lib()


def _dims(**kw):
    d = dict(dtype=0, steps=5, n_batch=2, rows=16, cols=24, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7, reserved=0)
    d.update(kw)
    return op.evo_orth_dims(*d.values())


def _orth(d, x=FAKE, out=FAKE + 0x100000, ws=FAKE + 0x1000000, ws_bytes=BIG):
    return _lib().evo_orthogonalize(ctypes.byref(d) if d is not None else None, x, out, ws, ws_bytes, None)


def test_exports_declared_symbols():
    text = open(os.path.join(ROOT, "include", "evo_muon.h")).read()
    for n in re.findall(r"^\s*(?:int|int64_t|size_t)\s*(evo_\w+)\s*\(", text, flags=re.M):
        assert hasattr(_lib(), n), n


BAD_COEFS = [(dict(a=float("nan")), 1), (dict(eps=0.0), 1), (dict(eps=float("inf")), 1), (dict(steps=0), 1),
             (dict(steps=65), 2), (dict(a=100.0), 2), (dict(a=3.0, b=0.0, c=0.0), 2), (dict(a=2.0, b=-70.0), 2)]


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(n_batch=-1), 1), (dict(rows=-1), 1), (dict(cols=-1), 1), (dict(rows=32769), 2),
    (dict(n_batch=(1 << 20) + 1), 2), (dict(n_batch=1 << 20, rows=32768, cols=32768), 2), (dict(reserved=1), 1),
] + BAD_COEFS)
def test_rejects_bad_dims(kw, status):
    assert _orth(_dims(**kw)) == status
    assert _lib().evo_orthogonalize_workspace_size(ctypes.byref(_dims(**kw))) == 0


def test_rejects_bad_pointers():
    d = _dims()
    need = _lib().evo_orthogonalize_workspace_size(ctypes.byref(d))
    assert need > 0
    assert _orth(None) == 1 and _orth(d, x=None) == 1 and _orth(d, out=None) == 1
    assert _orth(d, out=FAKE + 4) == 1                              # overlaps x
    assert _orth(d, x=FAKE + 2) == 3 and _orth(d, out=FAKE + 0x100002) == 3
    assert _orth(d, ws=None) == 4 and _orth(d, ws_bytes=need - 1) == 4 and _orth(d, ws=FAKE + 16) == 3
    for kw in (dict(n_batch=0), dict(rows=0), dict(cols=0)):
        assert _orth(_dims(**kw), x=None, out=None, ws=None, ws_bytes=0) == 0


def _tensors(shapes, **kw):
    t = np.zeros(len(shapes), dtype=np.dtype(op.evo_muon_tensor))
    for i, (r, c) in enumerate(shapes):
        v = dict(param=FAKE, grad=FAKE + 4096, momentum=FAKE + 8192, swa=0, rows=r, cols=c, update_scale=1.0)
        v.update(kw)
        t[i] = tuple(v.values())
    return t


def _plan(shapes, **kw):
    t = _tensors(shapes, **kw)
    n = _lib().evo_muon_plan_bytes(t.ctypes.data, len(t))
    plan = np.zeros(max(n, 8) // 8 + 1, dtype=np.int64)
    return t, n, plan


def test_plans():
    lib = _lib()
    t, n, plan = _plan([(16, 24), (0, 5), (200, 3), (65, 64)])
    assert n > 0 and lib.evo_muon_build_plan(t.ctypes.data, 4, plan.ctypes.data, n) == 0
    assert lib.evo_muon_workspace_size(plan.ctypes.data) > 0
    assert lib.evo_muon_build_plan(t.ctypes.data, 4, plan.ctypes.data, n - 1) == 4
    assert lib.evo_muon_build_plan(t.ctypes.data, 4, None, n) == 1
    assert lib.evo_muon_plan_bytes(None, 1) == -1 and lib.evo_muon_plan_bytes(t.ctypes.data, -1) == -1
    for bad in ((-1, 4), (4, 32769)):
        assert _plan([bad])[1] == -1
    for kw, st in ((dict(param=0), 1), (dict(grad=0), 1), (dict(momentum=0), 1), (dict(update_scale=float("inf")), 1),
                   (dict(param=FAKE + 2), 3), (dict(swa=FAKE + 1), 3)):
        t, n, plan = _plan([(4, 4)], **kw)
        assert lib.evo_muon_build_plan(t.ctypes.data, 1, plan.ctypes.data, n) == st, kw


def _hp(**kw):
    d = dict(lr=0.02, momentum=0.95, weight_decay=0.0, swa_decay=0.999, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7,
             steps=5, nesterov=1)
    d.update(kw)
    return op.evo_muon_hparams(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(lr=float("nan")), 1), (dict(momentum=1.0), 1), (dict(momentum=-0.1), 1), (dict(swa_decay=1.5), 1),
    (dict(weight_decay=float("inf")), 1), (dict(nesterov=2), 1)] + BAD_COEFS)
def test_step_rejects_bad_hparams(kw, status):
    lib = _lib()
    t, n, plan = _plan([(16, 24)])
    assert lib.evo_muon_build_plan(t.ctypes.data, 1, plan.ctypes.data, n) == 0
    assert lib.evo_muon_step(ctypes.byref(_hp(**kw)), plan.ctypes.data, FAKE, None, FAKE, BIG, None) == status


def test_step_rejects_bad_plans():
    lib = _lib()
    t, n, plan = _plan([(16, 24)])
    lib.evo_muon_build_plan(t.ctypes.data, 1, plan.ctypes.data, n)
    hp, need = _hp(), lib.evo_muon_workspace_size(plan.ctypes.data)
    st = lambda p=plan.ctypes.data, d=FAKE, g=None, w=FAKE, b=BIG, h=ctypes.byref(hp): lib.evo_muon_step(h, p, d, g, w, b, None)
    assert st(h=None) == 1 and st(p=None) == 1 and st(d=None) == 1
    assert st(g=FAKE + 2) == 3 and st(d=FAKE + 4) == 3 and st(w=FAKE + 16) == 3
    assert st(w=None) == 4 and st(b=need - 1) == 4
    other = np.zeros_like(plan)
    assert st(p=other.ctypes.data) == 1 and lib.evo_muon_workspace_size(other.ctypes.data) == 0
    t, n, plan0 = _plan([(0, 3)])
    assert lib.evo_muon_build_plan(t.ctypes.data, 1, plan0.ctypes.data, n) == 0
    assert st(p=plan0.ctypes.data, d=None, w=None, b=0) == 0         # nothing to do


def test_binding_refuses_before_any_launch():
    m = torch.zeros(4, 4)
    for x in (torch.zeros(4), torch.zeros(4, 4, dtype=torch.float16), torch.zeros(2, 2, 2, 2)):
        with pytest.raises(ValueError, match="matrix"):
            op.orthogonalize(x)
    with pytest.raises(ValueError, match="contiguous"):
        op.orthogonalize(m)
    with pytest.raises(ValueError, match="FusedAdamSWA"):
        op.FusedMuonSWA([torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(ValueError, match="one gradient"):
        op.FusedMuonSWA([m], [])
    with pytest.raises(ValueError, match="momentum"):
        op.FusedMuonSWA([m], [m], [m, m], [m])
    with pytest.raises(ValueError, match="adjust"):
        op.FusedMuonSWA([m], [m], adjust="other")
    with pytest.raises(ValueError, match="float32 CUDA"):
        op.FusedMuonSWA([m], [m])


def test_rejects_more_tiles_than_a_launch_takes():
    # 1 x 1300 is 21 tiles of 64 x 64: 2^20 of them are more than 2^24, and 2^19 are not
    assert _orth(_dims(n_batch=1 << 20, rows=1, cols=1300)) == 2
    assert _lib().evo_orthogonalize_workspace_size(ctypes.byref(_dims(n_batch=1 << 20, rows=1, cols=1300))) == 0
    assert _lib().evo_orthogonalize_workspace_size(ctypes.byref(_dims(n_batch=1 << 19, rows=1, cols=1300))) > 0
    # 64 of 32768 x 32768 are exactly 2^24
    assert _orth(_dims(n_batch=64, rows=32768, cols=32768)) == 2
    assert _plan([(32768, 32768)] * 64)[1] == -1


def test_coefficients_are_followed_through_the_steps():
    """The refusal against the largest singular value found on a fine grid, over coefficients of every kind."""
    rng = np.random.default_rng(0)
    kinds = {0: 0, 2: 0}
    for _ in range(400):
        a, b, c = rng.uniform(-4, 5), rng.choice([0.0, rng.uniform(-8, 8)]), rng.choice([0.0, rng.uniform(-4, 4)])
        steps, top, ok, near = int(rng.integers(1, 9)), 1.0, True, False
        for _ in range(steps):
            size = abs(a) + abs(b) * top ** 2 + abs(c) * top ** 4
            near |= abs(size - 60) < 1e-3 or abs(top - 8) < 1e-3
            ok &= top <= 8 and size <= 60
            if not ok:
                break
            s = np.linspace(0, top, 20001)
            top = np.abs(s * (a + s * s * (b + s * s * c))).max()
        near |= abs(top - 8) < 1e-3
        ok &= top <= 8
        if not near:
            kinds[0 if ok else 2] += 1
            assert _orth(_dims(a=a, b=b, c=c, steps=steps, n_batch=0)) == (0 if ok else 2), (a, b, c, steps, top)
    assert min(kinds.values()) > 50
