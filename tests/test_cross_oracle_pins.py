"""Pins of the oracle of attention to states of another length (CPU)."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co


def _inputs(seed, N=3, Lq=4, Lk=6, H=4, Hk=2, d=8, planes=3, mask=True):
    rng = np.random.default_rng(seed)
    q, dout, gate = (rng.standard_normal((N, Lq, H, d)) for _ in range(3))
    k, v = (rng.standard_normal((N, Lk, Hk, d)) for _ in range(2))
    bias = rng.standard_normal((planes, H, Lq, Lk)) if planes else None
    m = (rng.random((N, Lk)) < 0.7).astype(np.uint8) if mask else None
    if mask:
        m[:, 0] = 1
    return q, k, v, gate, bias, m, dout


@pytest.mark.parametrize("planes", [0, 1, 3])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_torch_autograd(planes, mask, gated):
    q, k, v, gate, bias, m, dout = _inputs(1, planes=planes, mask=mask)
    if not gated:
        gate = None
    N, Lq, H, d = q.shape
    rpb = N // planes if planes else None
    t = [None if x is None else torch.from_numpy(x).requires_grad_() for x in (q, k, v, gate, bias)]
    add = torch.zeros(N, H, Lq, k.shape[1], dtype=torch.float64)
    if planes:
        add = add + t[4].repeat_interleave(N // planes, 0)
    if mask:
        add = add.masked_fill(torch.from_numpy(m == 0)[:, None, None, :], -torch.inf)
    kk, vv = (x.permute(0, 2, 1, 3).repeat_interleave(2, 1) for x in t[1:3])
    a = torch.nn.functional.scaled_dot_product_attention(t[0].permute(0, 2, 1, 3), kk, vv, attn_mask=add).permute(0, 2, 1, 3)
    out = a * torch.sigmoid(t[3]) if gated else a
    (out * torch.from_numpy(dout)).sum().backward()
    o, lse, prob = co.forward(q, k, v, gate, bias, m, rpb)
    assert np.allclose(o, out.detach().numpy(), atol=1e-12)
    logits = np.einsum("nqhd,nkhd->nhqk", q, np.repeat(k, 2, 2)) / np.sqrt(d) + add.detach().numpy()
    assert np.allclose(lse, torch.logsumexp(torch.from_numpy(logits), 3).numpy(), atol=1e-12)
    got = co.backward(q, k, v, gate, bias, m, dout, rpb)
    for a, b in zip(got, t):
        assert (a is None) == (b is None)
        assert a is None or np.allclose(a, b.grad.numpy(), atol=1e-12)


def test_differences():
    q, k, v, gate, bias, m, dout = _inputs(2, planes=1)
    args = [q, k, v, gate, bias]
    grads = co.backward(q, k, v, gate, bias, m, dout)
    f = lambda *x: float(np.sum(co.forward(*x, m)[0] * dout))
    rng = np.random.default_rng(0)
    for i, g in enumerate(grads):
        for _ in range(4):
            at = tuple(rng.integers(0, n) for n in g.shape)
            lo, hi = [x.copy() for x in args], [x.copy() for x in args]
            lo[i][at] -= 1e-6
            hi[i][at] += 1e-6
            assert abs((f(*hi) - f(*lo)) / 2e-6 - g[at]) < 1e-7


def test_nothing_left_is_zero_and_masked_values_do_not_matter():
    q, k, v, gate, bias, m, dout = _inputs(3, planes=1)
    m[1] = 0
    ref = co.forward(q, k, v, gate, bias, m)
    assert not ref[0][1].any() and (ref[1][1] == -np.inf).all()
    gr = co.backward(q, k, v, gate, bias, m, dout)
    assert not gr[0][1].any() and not gr[1][1].any() and not gr[3][1].any()
    k2, v2 = k.copy(), v.copy()
    k2[m == 0], v2[m == 0] = np.nan, np.inf
    for a, b in zip(co.forward(q, k2, v2, gate, bias, m), ref):
        assert np.array_equal(a, b)
    assert not gr[2][m == 0].any()
    low = bias.copy()
    low[:, 1, 2] = -3.3895e38
    out, lse, _ = co.forward(q, k, v, gate, low, m)
    assert not out[:, 2, 1].any() and (lse[:, 1, 2] == -np.inf).all() and out[0, 1, 1].any()
    empty = co.forward(q, k[:, :0], v[:, :0])
    assert not empty[0].any() and (empty[1] == -np.inf).all()
