"""GPU parity of the gradients of the attention to states of another length
where logits lie far from zero at all keys of a query: its fp32 log-sum-exp no
longer holds the logarithm of the sum there, and its probabilities have to
come to one all the same.

Inputs and bounds as in the forward's tests of far logits: queries and keys on
different halves of the head, so that the logits are the biases, without any
rounding, and bounds at biases less the query's largest.
"""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paper_2404_11068_amd import cross
from tests.parity_util import to_f64
from tests.test_gpu_cross import F, _bounds, _close, _draw
from tests.test_gpu_cross_far_logits import _apart, _check_far, _same_keys

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
# tiles, the walked axis split over workgroups (queries and keys), many rows of the batch
SHAPES = [(2, 70, 77, 4, 2, 64), (2, 150, 200, 4, 4, 32), (1, 40, 3000, 2, 1, 128), (1, 1500, 90, 2, 2, 64), (40, 33, 50, 2, 2, 16)]
IDS = ["rows", "heads", "split", "queries", "batch"]


@DTYPES
@pytest.mark.parametrize("low", [-900.0, -1500.0, -4e4, -1e6, -1e7, -1e8, -1e9, -1e15, -0.9e30, -1.2e30, 3e3, 1e8])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_all_keys_far(shape, low, dtype):
    """Every other query has all its keys far off, equal (bf16) or a step or two of fp32 apart."""
    N, Lq, Lk, H, Hk, d = shape
    args = _draw((N, Lq, Lk, H, Hk, d, True, 1, "random"), dtype, 31)
    _apart(*args[:2])
    args[5][:] = args[5][:1]
    args[5][:, Lk // 2] = 1
    b = args[4][:, :, ::2]
    b[:] = low
    if dtype == torch.float32 and abs(low) < 1e9:
        step = max(float(np.spacing(np.float32(abs(low)))), 0.25)
        b += step * torch.randint(-2, 3, b.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
    _check_far(args)


@DTYPES
def test_far_and_ordinary_planes(dtype):
    """A bias plane for every row of the batch, one of them far off throughout, heads of their own range, some keys masked
    by the bias; and the gradients' bits do not change between calls."""
    N, Lq, Lk, H, d = 3, 45, 130, 3, 32
    args = _draw((N, Lq, Lk, H, H, d, False, N, None), dtype, 32)
    _apart(*args[:2])
    args[4][1] = -1e9
    args[4][0, 1] = -1e5
    args[4][2, 2] = 1e7
    args[4][2, 2, :, ::3] = -float("inf")
    args[4][0, 0, :, 5:60] = -1e9
    _check_far(args, rpb=1)
    q, k, v, g, bias, m, dout = args
    out, lse = cross.cross_attn_fwd(q, k, v, g, bias, rows_per_bias=1)
    one, two = (cross.cross_attn_bwd(q, k, v, g, bias, None, out, lse, dout, rows_per_bias=1) for _ in range(2))
    for a, b in zip(one, two):
        assert a is None or torch.equal(a, b)


@DTYPES
@pytest.mark.parametrize("size", [3e3, 1e6, -1e7, 1e10, -3e10, -1.1e15])
@pytest.mark.parametrize("N,Lq,Lk,H,d", [(2, 70, 301, 2, 32), (1, 40, 3000, 1, 128), (1, 1500, 60, 1, 64)],
                         ids=["rows", "keys", "queries"])
def test_gradients_at_far_products(N, Lq, Lk, H, d, size, dtype):
    """Without a bias: products of queries and keys far from zero and the same for all keys.  The channel that makes them is
    left out of the bounds' queries; its dK is the other side's channel of ones times it, its dQ a sum over
    keys of what comes to zero."""
    args = _same_keys(N, Lq, Lk, H, d, size, dtype, 33)
    q, k, v, _, _, _, dout = args
    u = 2.0 ** -8 if dtype == torch.bfloat16 else F
    out, lse = cross.cross_attn_fwd(q, k, v)
    grads = cross.cross_attn_bwd(q, k, v, None, None, None, out, lse, dout)[:3]
    torch.cuda.synchronize()
    f = [to_f64(t) for t in (q, k, v)]
    far = f[0][0, 0, 0, 0]
    want = co.backward(*f, None, None, None, to_f64(dout))[:3]
    near = [f[0].copy()] + f[1:]
    near[0][..., 0] = 0.0
    b = _bounds(*near, None, None, None, to_f64(dout), N, u)[2:5]
    b[1][..., 0] = abs(far) * b[1][..., -1]
    for name, got, r, bound in zip(("dq", "dk", "dv"), grads, want, b):
        _close(got, r, bound, u, name)


@DTYPES
@pytest.mark.parametrize("gate", [False, True], ids=["plain", "gate"])
@pytest.mark.parametrize("N,Lq,Lk,H,Hk,d", [(3, 45, 70, 6, 2, 40), (1, 20, 2100, 2, 1, 104)], ids=["rows", "split"])
def test_strided_tensors_far_and_near(N, Lq, Lk, H, Hk, d, gate, dtype):
    """Views of packed buffers, tokens outermost, with a bias that puts every third query far off: the bits of tensors of
    their own, a workspace of just the size asked for (nothing behind it is touched), and gradients in packed buffers."""
    q, k, v, g, bias, _, dout = _draw((N, Lq, Lk, H, Hk, d, gate, 1, None), dtype, 34)
    bias[:, :, ::3] = -1e9
    out, lse = cross.cross_attn_fwd(q, k, v, g, bias)
    want = cross.cross_attn_bwd(q, k, v, g, bias, None, out, lse, dout)
    qg = torch.zeros(Lq, N, 2 * H, d, dtype=dtype, device="cuda").transpose(0, 1)
    kv = torch.zeros(Lk, N, 2 * Hk, d, dtype=dtype, device="cuda").transpose(0, 1)
    od = torch.zeros(Lq, N, 3 * H, d, dtype=dtype, device="cuda").transpose(0, 1)
    qv, gv, kv_, vv, ov, dv_ = qg[:, :, :H], qg[:, :, H:], kv[:, :, :Hk], kv[:, :, Hk:], od[:, :, :H], od[:, :, 2 * H:]
    for to, x in ((qv, q), (kv_, k), (vv, v), (dv_, dout)) + (((gv, g),) if gate else ()):
        to.copy_(x)
    o2, l2 = cross.cross_attn_fwd(qv, kv_, vv, gv if gate else None, bias, out=ov)
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    need = cross.cross_attn_bwd_workspace_size(q, k, gate, True)
    room = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    dqg, dkv = torch.full_like(qg, 7.0), torch.full_like(kv, 7.0)
    kw = dict(dgate=dqg[:, :, H:]) if gate else {}
    got = cross.cross_attn_bwd(qv, kv_, vv, gv if gate else None, bias, None, ov, lse, dv_, dq=dqg[:, :, :H], dk=dkv[:, :, :Hk],
                               dv=dkv[:, :, Hk:], workspace=room[:need], **kw)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert a is None or torch.equal(a, b)
    assert (room[need:] == 171).all() and (gate or (dqg[:, :, H:] == 7.0).all())
