"""GPU parity of rotary positions and the norm of heads with the rotation
(through the C ABI) against the fp64 oracle.

Tolerances, in units of e = 2^-24 (half a step of fp32).  The angle is off by
2^-32 turns (1.5e-9) before it is rounded to fp32 (e of at most pi / 4) and
scaled (e); sine and cosine are series of a few fused steps, each rounding
at most e of a value up to 1, and the amplitude one more: 8 e covers angle
and series.  A rotated value is two products of them and one sum: with u the
pair's values, (8 + 2) e A (|u_a| + |u_b|), so 12 e A (|u_a| + |u_b|).
The norm: a sum of d squares, d e relative at most, halved by the root, and
four roundings of division, root and products: u is off by (d / 2 + 6) e |u|.
Backward: g as above, t = g w; mean(t xhat) sums d products, each off by
(d / 2 + 20) e, over d terms: (3 d / 2 + 30) e mean |t xhat|.  dw: n terms in
fp32, each off by the same, in parts whose sums round n e at most.
Results are rounded once more: 2^-8 (bf16) or e of the value.
"""
import numpy as np
import pytest
import torch

from oracle import rope_oracle as ro
from paper_2404_11068_amd import evo_attn as ea
from paper_2404_11068_amd import graph as gr
from paper_2404_11068_amd import rope
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def _rand(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape)).to(dtype).cuda()


def _half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E


def _abs_pair(u, rot, interleaved):
    """|u_a| + |u_b| at both channels of each pair, |u| elsewhere."""
    m = np.abs(u).copy()
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    s = m[..., a] + m[..., b]
    m[..., a], m[..., b] = s, s
    return m


def _check(got, ref, bound, dtype):
    off = np.abs(to_f64(got) - ref)
    limit = bound + _half(dtype) * (np.abs(ref) + bound) + 2.0 ** -130
    assert (off <= limit).all(), (float((off / limit).max()), np.unravel_index((off / limit).argmax(), off.shape))


CASES = [
    # N, Lq, Lk, H, Hk, d, rot, interleaved, far
    (1, 1, 0, 1, 0, 8, 8, False, 0),
    (3, 1, 1, 8, 2, 128, 128, False, 100000),
    (2, 5, 9, 3, 1, 64, 64, False, 0),
    (2, 7, 3, 4, 4, 64, 32, True, 2 ** 30),
    (1, 33, 70, 5, 5, 32, 24, False, 1000),
    (2, 17, 1, 6, 2, 40, 20, False, 0),
    (1, 9, 9, 2, 1, 256, 250, False, 12345),
    (4, 3, 11, 7, 7, 96, 96, True, 0),
    (1, 40, 3, 1, 1, 8, 2, False, 0),
    (1, 40, 3, 1, 1, 16, 0, False, 0),
    (2, 1200, 601, 2, 1, 16, 16, False, 5),
    (130, 17, 33, 1, 1, 24, 24, True, 0),
]


def _inputs(case, dtype, seed):
    N, Lq, Lk, H, Hk, d, rot, inter, far = case
    rng = np.random.default_rng(seed)
    sets = []
    for L, h in ((Lq, H), (Lk, Hk)):
        if not h:
            sets.append((None,) * 4)
            continue
        pos = (far + rng.integers(-3, 1000, (N, 1)) + np.arange(L)).astype(np.int32)
        w = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).cuda()
        sets.append((_rand(rng, (N, L, h, d), dtype), _rand(rng, (N, L, h, d), dtype), torch.from_numpy(pos).cuda(), w))
    freq = rope.rope_frequencies(rot)
    return sets, freq, rope.rope_steps(freq), rng


@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "N%d_%dx%d_H%d_%d_d%d_r%d_%s_%d" % c)
def test_forward_and_backward(case, dtype, norm):
    print("\n[case]", case, dtype, norm, flush=True)
    N, Lq, Lk, H, Hk, d, rot, inter, far = case
    (q, dq, pq, wq), (k, dk, pk, wk) = _inputs(case, dtype, 1)[0]
    freq, steps = _inputs(case, dtype, 1)[1:3]
    amp, eps = 1.125, 1e-5
    kw = dict(interleaved=inter, amplitude=amp, pos_k=pk, norm=norm, eps=eps)
    if norm:
        kw.update(weight_q=wq, weight_k=wk)
    out = rope.rope_fwd(q, pq, steps, k=k, **kw)
    bkw = dict(kw, q=q, k=k) if norm else kw
    grad = rope.rope_bwd(dq, pq, steps, dk=dk, **bkw)
    again = rope.rope_bwd(dq, pq, steps, dk=dk, **bkw)
    torch.cuda.synchronize()
    for i, (x, dy, pos, w) in enumerate(((q, dq, pq, wq), (k, dk, pk, wk))):
        if x is None:
            assert out[i] is None and grad[i] is None and grad[i + 2] is None
            continue
        x64, dy64, p64, w64 = to_f64(x), to_f64(dy), pos.cpu().numpy(), to_f64(w) if norm else None
        okw = dict(interleaved=inter, amplitude=amp, norm=norm, w=w64, eps=eps)
        u = x64 * ro.rstd(x64, eps) * w64 if norm else x64
        rel = (d / 2 + 6) * E if norm else 0.0
        _check(out[i], ro.forward(x64, p64, freq, **okw), (12 * E * amp + rel * amp) * _abs_pair(u, rot, inter) + rel * np.abs(u), dtype)
        dx, dw = ro.backward(dy64, x64, p64, freq, **okw)
        bound = 12 * E * amp * _abs_pair(dy64, rot, inter)
        if norm:
            r = ro.rstd(x64, eps)
            g = amp * _abs_pair(dy64, rot, inter)      # bounds |g|
            hat, t = np.abs(x64 * r), g * np.abs(w64)
            n = 1.5 * d + 30
            bound = n * E * r * (t + 2 * hat * np.mean(t * hat, -1, keepdims=True))
            count = x64.shape[0] * x64.shape[1] * x64.shape[2]
            assert (np.abs(to_f64(grad[i + 2]) - dw) <= (n + count) * E * np.sum(g * hat, (0, 1, 2))).all()
            assert torch.equal(grad[i + 2], again[i + 2])
        _check(grad[i], dx, bound, dtype)
        assert torch.equal(grad[i], again[i])


def test_far_positions_of_both_signs():
    """The ends of int32: the phase is an integer product, no argument is too large for it."""
    ends = [-2 ** 31, -2 ** 31 + 1, -65537, -1, 0, 1, 2 ** 24 + 1, 2 ** 31 - 1]
    pos = torch.tensor([ends], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    x = _rand(rng, (1, 8, 2, 64), torch.float32)
    freq = rope.rope_frequencies(64)
    out, _ = rope.rope_fwd(x, pos, rope.rope_steps(freq))
    x64 = to_f64(x)
    # the table of steps is off by 2^-65 turns a position: 2^-34 turns, 3.7e-10, and extended precision by 2^-32
    bound = (12 * E + 1e-9) * _abs_pair(x64, 64, False)
    _check(out, ro.forward(x64, pos.cpu().numpy(), freq), bound, torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_views_of_packed_projections_in_place_and_shared_positions(dtype):
    rng = np.random.default_rng(4)
    N, L, H, Hk, d = 2, 21, 4, 2, 32
    packed = _rand(rng, (N, L, H + 2 * Hk, d), dtype)
    q, k, v = packed[:, :, :H], packed[:, :, H:H + Hk], packed[:, :, H + Hk:]
    pos = torch.arange(L, dtype=torch.int32, device="cuda")
    steps = rope.rope_steps(rope.rope_frequencies(d))
    w = torch.rand(d, device="cuda") + 0.5
    kw = dict(norm=True, weight_q=w)
    ref = rope.rope_fwd(q.contiguous(), pos.expand(N, L).contiguous(), steps, k=k.contiguous(), pos_k=pos.view(1, L), **kw)
    before = packed.clone()
    dq, dk = torch.randn_like(ref[0]), torch.randn_like(ref[1])
    g_ref = rope.rope_bwd(dq, pos, steps, dk=dk, pos_k=pos, q=q.contiguous(), k=k.contiguous(), **kw)
    g = rope.rope_bwd(dq, pos, steps, dk=dk, pos_k=pos, q=q, k=k, **kw)
    torch.cuda.synchronize()
    assert g[0].stride() == q.stride()
    for a, b in zip(g, g_ref):
        assert (a is None and b is None) or torch.equal(a, b)
    got = rope.rope_fwd(q, pos, steps, k=k, pos_k=pos, out_q=q, out_k=k, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert torch.equal(v, before[:, :, H + Hk:])                       # what lies between stays
    # rows and tokens swapped: a transposed view
    x = _rand(rng, (L, N, H, d), dtype)
    a, _ = rope.rope_fwd(x.transpose(0, 1), pos, steps)
    b, _ = rope.rope_fwd(x.transpose(0, 1).contiguous(), pos, steps)
    assert torch.equal(a, b)
    # one row for all
    one = x[:, :1].transpose(0, 1)
    a, _ = rope.rope_fwd(one.expand(3, L, H, d), torch.stack([pos, pos + 5, pos - 900]), steps)
    b, _ = rope.rope_fwd(one.repeat(3, 1, 1, 1), torch.stack([pos, pos + 5, pos - 900]), steps)
    assert torch.equal(a, b)
    # backward of the rotation undoes it, in place
    y, _ = rope.rope_fwd(x.transpose(0, 1).contiguous().float(), pos, steps)
    z = y.clone()
    got = rope.rope_bwd(z, pos, steps, out_q=z)[0]
    assert got is z and float((z - x.transpose(0, 1).float()).abs().max()) < 1e-5


def test_captured_calls_and_other_streams():
    rng = np.random.default_rng(5)
    q, k = _rand(rng, (2, 50, 4, 64), torch.bfloat16), _rand(rng, (2, 70, 2, 64), torch.bfloat16)
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    pq, pk = torch.arange(50, dtype=torch.int32, device="cuda"), torch.arange(70, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    steps = rope.rope_steps(rope.rope_frequencies(64))
    kw = dict(norm=True, weight_q=w, weight_k=w)
    ws = torch.empty(rope.rope_bwd_workspace_size(q, steps, k=k, norm=True), dtype=torch.uint8, device="cuda")
    oq, ok, gq, gk = (torch.empty_like(t) for t in (q, k, q, k))
    wq, wk = torch.empty_like(w), torch.empty_like(w)

    def record(stream):
        rope.rope_fwd(q, pq, steps, k=k, pos_k=pk, out_q=oq, out_k=ok, stream=stream, **kw)
        rope.rope_bwd(dq, pq, steps, dk=dk, pos_k=pk, q=q, k=k, out_q=gq, out_k=gk, dweight_q=wq, dweight_k=wk,
                      workspace=ws, stream=stream, **kw)

    s, cache = torch.cuda.Stream(), gr.GraphCache(capacity=2)
    for replay in range(4):
        for t in (q, k, dq, dk):
            t.normal_()
        w.uniform_(0.5, 1.5)
        torch.cuda.synchronize()
        cache.run(7, record, s)
        torch.cuda.synchronize()
        ref = rope.rope_fwd(q, pq, steps, k=k, pos_k=pk, **kw) + \
            rope.rope_bwd(dq, pq, steps, dk=dk, pos_k=pk, q=q, k=k, **kw)
        torch.cuda.synchronize()
        for a, b in zip((oq, ok, gq, gk, wq, wk), ref):
            assert torch.equal(a, b)


def test_refuses():
    q = torch.zeros(2, 4, 2, 16, device="cuda", dtype=torch.bfloat16)
    p = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    s = torch.zeros(8, dtype=torch.int64, device="cuda")
    w = torch.ones(16, device="cuda")
    bad = [dict(pos_q=p.long()), dict(pos_q=p[:, :3]), dict(pos_q=p.cpu()), dict(steps=s.int()), dict(steps=torch.zeros(9, dtype=torch.int64, device="cuda")),
           dict(weight_q=w), dict(norm=True, weight_q=w[:8]), dict(norm=True, weight_q=w.bfloat16()), dict(k=q.float(), pos_k=p),
           dict(k=q), dict(k=q[:1], pos_k=p), dict(pos_k=p), dict(out_q=q[:, :3]), dict(out_k=q), dict(out_q=q.float())]
    for kw in bad:
        args = dict(q=q, pos_q=p, steps=s)
        args.update(kw)
        with pytest.raises(ValueError):
            rope.rope_fwd(**args)
    with pytest.raises(ea.EvoAttnError):
        rope.rope_fwd(q, p, s, norm=True, eps=-1.0)
    with pytest.raises(ea.EvoAttnError):
        rope.rope_fwd(q, p, s, out_q=q[:1].expand(2, 4, 2, 16))      # an output that overlaps itself
    with pytest.raises(ea.EvoAttnError):
        rope.rope_bwd(q, p, s, norm=True, q=q, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_an_eps_of_zero(dtype):
    """Lanes without a unit must not count: nothing over the root of nothing."""
    rng = np.random.default_rng(6)
    q, dq = _rand(rng, (1, 5, 3, 40), dtype), _rand(rng, (1, 5, 3, 40), dtype)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    freq = rope.rope_frequencies(40)
    w = torch.ones(40, device="cuda")
    g = rope.rope_bwd(dq, pos, rope.rope_steps(freq), q=q, norm=True, weight_q=w, eps=0.0)
    dx, dw = ro.backward(to_f64(dq), to_f64(q), np.arange(5)[None], freq, norm=True, w=np.ones(40), eps=0.0)
    hat = np.abs(to_f64(q)) * ro.rstd(to_f64(q), 0.0)
    bound = (1.5 * 40 + 30 + 15) * E * np.sum(_abs_pair(to_f64(dq), 40, False) * hat, (0, 1, 2))
    assert (np.abs(to_f64(g[2]) - dw) <= bound).all() and g[0].isfinite().all()


def test_empty_sets():
    s = rope.rope_steps(rope.rope_frequencies(16))
    w = torch.ones(16, device="cuda")
    q = torch.zeros(2, 0, 2, 16, device="cuda")
    k = torch.randn(2, 3, 2, 16, device="cuda")
    p0, p3 = torch.zeros(2, 0, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    oq, ok = rope.rope_fwd(q, p0, s, k=k, pos_k=p3)
    assert oq.shape == q.shape and torch.equal(ok, k)                  # position 0 turns nothing
    dw = torch.full((16,), 7.0, device="cuda")
    g = rope.rope_bwd(q, p0, s, dk=k, pos_k=p3, q=q, k=k, norm=True, weight_q=w, weight_k=w, dweight_q=dw)
    torch.cuda.synchronize()
    assert g[2] is dw and not dw.any() and g[3].isfinite().all()
    g = rope.rope_bwd(k[:0], p3[:0], s, q=k[:0], norm=True, weight_q=w, dweight_q=dw.fill_(3.0))
    torch.cuda.synchronize()
    assert not dw.any()


@pytest.mark.parametrize("rot", [64, 48, 40], ids=["whole", "part", "odd"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
def test_gradients_in_the_place_of_their_heads(rot, interleaved):
    # with the norm dx may be written over x, or over dy: the same bits as into tensors of its own
    rng = np.random.default_rng(11)
    dt = torch.bfloat16
    q, dq = (torch.tensor(rng.standard_normal((3, 517, 5, 64)), dtype=dt, device="cuda") for _ in range(2))
    k, dk = (torch.tensor(rng.standard_normal((3, 33, 2, 64)), dtype=dt, device="cuda") for _ in range(2))
    w = torch.tensor(rng.standard_normal(64), dtype=torch.float32, device="cuda")
    pos = torch.arange(517, dtype=torch.int32, device="cuda")
    steps = rope.rope_steps(rope.rope_frequencies(rot))
    kw = dict(pos_k=pos[:33], norm=True, interleaved=interleaved, weight_q=w, weight_k=w)
    want = rope.rope_bwd(dq, pos, steps, dk=dk, q=q, k=k, **kw)
    q2, k2, dq2, dk2 = (t.clone() for t in (q, k, dq, dk))
    over_x = rope.rope_bwd(dq, pos, steps, dk=dk, q=q2, k=k2, out_q=q2, out_k=k2, **kw)
    over_dy = rope.rope_bwd(dq2, pos, steps, dk=dk2, q=q, k=k, out_q=dq2, out_k=dk2, **kw)
    for a, b, c in zip(want, over_x, over_dy):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert torch.equal(want[0], q2) and torch.equal(want[1], dk2)
