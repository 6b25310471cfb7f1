"""Host-side checks of the rotary positions (no GPU): exports, every invalid
call rejected before any HIP call (fake addresses never touched), and the
binding's refusals."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2404_11068_amd import evo_attn as ea
from paper_2404_11068_amd import rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000
BIG = 0x10000000
P = lambda x: None if x is None else ctypes.c_void_p(x)


def _lib():
    if not os.path.exists(ea.LIB_PATH):
        pytest.skip("libevoattn.so not built")
    return rope._lib()


def _dims(**kw):
    d = dict(dtype=1, head_dim=64, rot_dim=64, flags=2, n_heads=(8, 2), eps=1e-6, amplitude=1.0, n_rows=2, len=(16, 24),
             pos_stride=(16, 24), x_stride_row=(16 * 512, 24 * 128), x_stride_tok=(512, 128),
             y_stride_row=(16 * 512, 24 * 128), y_stride_tok=(512, 128))
    d.update(kw)
    return rope.evo_rope_dims(*[x for v in d.values() for x in (v if isinstance(v, tuple) else (v,))])


def _fwd(d, x0=FAKE, x1=FAKE + BIG, pos0=FAKE + 2 * BIG, pos1=FAKE + 3 * BIG, steps=FAKE + 4 * BIG, w0=FAKE + 5 * BIG,
         w1=FAKE + 6 * BIG, y0=FAKE + 7 * BIG, y1=FAKE + 8 * BIG):
    return _lib().evo_rope_fwd(ctypes.byref(d) if d is not None else None, P(x0), P(x1), P(pos0), P(pos1), P(steps),
                               P(w0), P(w1), P(y0), P(y1), None)


def _bwd(d, dy0=FAKE + 9 * BIG, dy1=FAKE + 10 * BIG, x0=FAKE, x1=FAKE + BIG, pos0=FAKE + 2 * BIG, pos1=FAKE + 3 * BIG,
         steps=FAKE + 4 * BIG, w0=FAKE + 5 * BIG, w1=FAKE + 6 * BIG, dx0=FAKE + 7 * BIG, dx1=FAKE + 8 * BIG,
         dw0=FAKE + 11 * BIG, dw1=FAKE + 12 * BIG, ws=FAKE + 13 * BIG, ws_bytes=1 << 40):
    return _lib().evo_rope_bwd(ctypes.byref(d) if d is not None else None, P(dy0), P(dy1), P(x0), P(x1), P(pos0), P(pos1),
                               P(steps), P(w0), P(w1), P(dx0), P(dx1), P(dw0), P(dw1), P(ws), ws_bytes, None)


def test_exports_declared_symbols():
    text = open(os.path.join(ROOT, "include", "evo_rope.h")).read()
    names = re.findall(r"^\s*(?:int|size_t)\s*(evo_\w+)\s*\(", text, flags=re.M)
    assert len(names) == 3
    for n in names:
        assert hasattr(_lib(), n), n


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(head_dim=0), 1), (dict(head_dim=12, rot_dim=8), 2), (dict(head_dim=264), 2),
    (dict(rot_dim=66), 1), (dict(rot_dim=3), 1), (dict(rot_dim=-2), 1), (dict(flags=4), 1), (dict(n_heads=(0, 2)), 1),
    (dict(n_heads=(8, -1)), 1), (dict(n_heads=(65536, 2)), 2), (dict(n_rows=-1), 1), (dict(len=(-1, 24)), 1),
    (dict(len=((1 << 30) + 1, 24)), 2), (dict(n_rows=1 << 40), 2), (dict(pos_stride=(-1, 0)), 1), (dict(eps=-1.0), 1),
    (dict(eps=math.nan), 1), (dict(eps=math.inf), 1), (dict(amplitude=math.inf), 1), (dict(amplitude=math.nan), 1),
    (dict(x_stride_tok=(-512, 128)), 1), (dict(x_stride_tok=(516, 128), y_stride_tok=(516, 128)), 3),
    (dict(x_stride_tok=(256, 128), y_stride_tok=(256, 128)), 1),
    (dict(x_stride_row=(1 << 41, 24 * 128)), 2), (dict(pos_stride=(1 << 41, 24)), 2),
    (dict(x_stride_row=(512, 24 * 128), y_stride_row=(512, 24 * 128)), 1),
    (dict(x_stride_row=(16 * 512, 0), y_stride_row=(16 * 512, 0)), 1),
])
def test_rejects_bad_dims(kw, status):
    d = _dims(**kw)
    assert _fwd(d) == status and _bwd(d) == status
    assert _lib().evo_rope_bwd_workspace_size(ctypes.byref(d)) == 0


def test_inputs_may_repeat_but_not_outputs():
    """x of row stride 0 is one row for all; y, and dx with x's strides, must not overlap themselves."""
    d = _dims(x_stride_row=(0, 0))
    assert _bwd(d) == 1
    assert _fwd(_dims(y_stride_row=(0, 24 * 128))) == 1


def test_rejects_bad_pointers():
    d = _dims()
    assert _fwd(None) == 1 and _bwd(None) == 1
    for k in ("x0", "x1", "pos0", "pos1", "steps", "y0", "y1"):
        assert _fwd(d, **{k: None}) == 1, k
    for k in ("dy0", "dy1", "x0", "x1", "pos0", "pos1", "steps", "dx0", "dx1", "dw0", "dw1", "w0", "w1"):
        assert _bwd(d, **{k: None}) == 1, k
    for k in ("x0", "x1", "y0", "y1"):
        assert _fwd(d, **{k: FAKE + 20 * BIG + 8}) == 3, k
    for k, off in (("pos0", 2), ("steps", 4), ("w1", 2)):
        assert _fwd(d, **{k: FAKE + 20 * BIG + off}) == 3, k
    for k, off in (("dy0", 8), ("x1", 8), ("dx1", 8), ("dw0", 2), ("pos1", 1), ("ws", 8)):
        assert _bwd(d, **{k: FAKE + 20 * BIG + off}) == 3, k
    plain = _dims(flags=0)
    assert _fwd(plain) == 1 and _bwd(plain) == 1                      # weights without the norm
    assert _fwd(d, y0=FAKE + 512) == 1 and _fwd(d, y0=FAKE - 512) == 1  # overlaps x, not in place
    assert _fwd(d, y1=FAKE + 7 * BIG) == 1                            # both outputs in one place
    assert _bwd(d, dx0=FAKE + 9 * BIG + 512) == 1 and _bwd(d, dw1=FAKE + 11 * BIG) == 1
    other = _dims(y_stride_row=(16 * 1024, 24 * 128), y_stride_tok=(1024, 128))
    assert _fwd(other, y0=FAKE) == 1                                  # same address, other strides
    need = _lib().evo_rope_bwd_workspace_size(ctypes.byref(d))
    assert need > 0 and _bwd(d, ws=None) == 4 and _bwd(d, ws_bytes=need - 1) == 4
    assert _lib().evo_rope_bwd_workspace_size(ctypes.byref(plain)) == 0


def test_sets_must_not_overlap_but_in_a_packed_buffer():
    d = _dims()
    assert _fwd(d, y0=FAKE + BIG) == 1 and _fwd(d, y1=FAKE) == 1              # on the other set's input
    assert _fwd(d, y1=FAKE + 7 * BIG + 256) == 1
    assert _bwd(d, dx0=FAKE + 10 * BIG) == 1 and _bwd(d, dx1=FAKE + 9 * BIG + 1024) == 1 and _bwd(d, dx1=FAKE) == 1
    # keys on the queries' last head in a packed buffer of tokens of 640 elements
    p = dict(len=(16, 16), x_stride_row=(16 * 640, 16 * 640), x_stride_tok=(640, 640), y_stride_row=(16 * 640, 16 * 640),
             y_stride_tok=(640, 640))
    assert _fwd(_dims(**p), y0=FAKE + 7 * BIG, y1=FAKE + 7 * BIG + 2 * 448) == 1


def test_empty_needs_no_pointers():
    none = {k: None for k in ("x0", "x1", "pos0", "pos1", "steps", "w0", "w1", "y0", "y1")}
    assert _fwd(_dims(n_rows=0), **none) == 0
    assert _fwd(_dims(len=(0, 0)), **none) == 0


def test_binding_refuses_before_any_launch():
    x, p = torch.zeros(2, 4, 2, 16), torch.zeros(2, 4, dtype=torch.int32)
    s, w = torch.zeros(8, dtype=torch.int64), torch.ones(16)
    bad = [
        (dict(q=x[0]), "N, L, H, d"), (dict(q=x.double()), "float32 or bfloat16"),
        (dict(q=torch.zeros(2, 4, 2, 32)[..., ::2]), "contiguous"), (dict(), "CUDA"),
    ]
    for kw, what in bad:
        args = dict(q=x, pos_q=p, steps=s, norm=True, weight_q=w)
        args.update(kw)
        with pytest.raises(ValueError, match=what):
            rope.rope_fwd(**args)
    with pytest.raises(ValueError, match="needs q"):
        rope.rope_bwd(x, p, s, norm=True)
    with pytest.raises(ValueError, match="go with norm"):
        rope.rope_bwd(x, p, s, q=x)
    with pytest.raises(ValueError, match="shaped like"):
        rope.rope_bwd(x, p, s, q=x[:1], norm=True)


def test_gradients_must_not_lie_across_their_inputs():
    # with the norm dx may be x itself, or apart from it; the missing workspace shows that a call goes on
    d = _dims()
    assert _bwd(d, dx0=FAKE, ws=None) == 4 and _bwd(d, dx1=FAKE + BIG, ws=None) == 4
    assert _bwd(d, dx0=FAKE + 16) == 1 and _bwd(d, dx1=FAKE + BIG + 128 * 2) == 1
    assert _bwd(d, dx0=FAKE + 2 * 16 * 512 * 2 - 16) == 1 and _bwd(d, dx0=FAKE + 2 * 16 * 512 * 2, ws=None) == 4
