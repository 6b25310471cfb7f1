"""GPU parity of the norm of heads where squares leave fp32's range: heads
whose channels' squares are denormal, vanish or overflow, beside ordinary ones.

Bounds as in the parity tests of the ordinary range; the oracle's fp64 holds
all of these squares.
"""
import numpy as np
import pytest
import torch

from oracle import rope_oracle as ro
from paper_2404_11068_amd import rope
from tests.parity_util import to_f64
from tests.test_gpu_rope import E, _abs_pair, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-6])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (40, False), (30, True), (0, False)],
                         ids=["half", "interleaved", "split", "part", "none"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_heads_of_any_magnitude(dtype, rot, interleaved, eps):
    rng = np.random.default_rng(41)
    N, L, H, d = 2, 37, 3, 64
    # heads of one size each, from denormal squares over ordinary ones to overflowing ones; gradients such that
    # what comes out is held in the type
    size = 10.0 ** rng.choice([-30.0, -25.0, -21.0, -19.5, -19.0, -18.0, 0.0, 0.0, 18.0, 18.7, 19.2, 20.0, 25.0, 30.0], (N, L, H, 1))
    x = torch.from_numpy(rng.standard_normal((N, L, H, d)) * size).to(dtype).cuda()
    x64 = to_f64(x)
    dy = torch.from_numpy(rng.standard_normal((N, L, H, d)) * np.minimum(1.0, np.sqrt(np.mean(x64 * x64, -1, keepdims=True) + eps) * 1e3)).to(dtype).cuda()
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).cuda()
    pos = torch.arange(L, dtype=torch.int32, device="cuda")
    freq = rope.rope_frequencies(rot)
    kw = dict(norm=True, weight_q=w, eps=eps, interleaved=interleaved)
    out, _ = rope.rope_fwd(x, pos, rope.rope_steps(freq), **kw)
    dx, _, dw, _ = rope.rope_bwd(dy, pos, rope.rope_steps(freq), q=x, **kw)
    torch.cuda.synchronize()
    dy64, w64, p = to_f64(dy), to_f64(w), np.broadcast_to(np.arange(L), (N, L))
    eps32 = float(np.float32(eps))
    okw = dict(interleaved=interleaved, norm=True, w=w64, eps=eps32)
    r = ro.rstd(x64, eps32)
    u = x64 * r * w64
    rel = (d / 2 + 6) * E
    _check(out, ro.forward(x64, p, freq, **okw), (12 * E + rel) * _abs_pair(u, rot, interleaved) + rel * np.abs(u), dtype)
    want, wdw = ro.backward(dy64, x64, p, freq, **okw)
    g = _abs_pair(dy64, rot, interleaved)
    hat, t = np.abs(x64 * r), g * np.abs(w64)
    n = 1.5 * d + 30
    _check(dx, want, 12 * E * g + n * E * r * (t + 2 * hat * np.mean(t * hat, -1, keepdims=True)), dtype)
    assert (np.abs(to_f64(dw) - wdw) <= (n + N * L * H) * E * np.sum(g * hat, (0, 1, 2))).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_heads_of_zeros(dtype):
    """With an eps: zeros stay zeros, whatever it is, and their gradients are finite."""
    x = torch.zeros(2, 5, 2, 32, device="cuda", dtype=dtype)
    dy = torch.ones_like(x)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    steps, w = rope.rope_steps(rope.rope_frequencies(32)), torch.ones(32, device="cuda")
    for eps in (1e-30, 1e-6):
        out, _ = rope.rope_fwd(x, pos, steps, norm=True, weight_q=w, eps=eps)
        dx, _, dw, _ = rope.rope_bwd(dy, pos, steps, q=x, norm=True, weight_q=w, eps=eps)
        torch.cuda.synchronize()
        g = ro.rotate(np.ones(x.shape), np.arange(5)[None].repeat(2, 0), rope.rope_frequencies(32), False, 1.0, True)
        assert not out.any() and not dw.any()
        r = 1 / np.sqrt(float(np.float32(eps)))
        _check(dx, g * r, 60 * E * 2 * r, dtype)
