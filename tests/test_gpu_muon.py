"""GPU parity of the Newton-Schulz orthogonalisation and the Muon step
(through the C ABI) against the fp64 oracle.

Tolerances, normwise over a matrix (Frobenius).  A step's rounding of
relative size e in X, A = X X^T, A A, P and P X changes the iterate by at most
C e |X| with C = 10 (|a| + 2 |b| |A| + 4 |c| |A|^2 around |A| <= 1.5, divided by the
gain of the step, and the five roundings); what a later step makes of the change
is bounded by its slope, 3.4445 at most.
  * Flat spectra (all singular values within a few times each other): the
    iterate grows along with the change, so the changes add up over the five
    steps: 5 C e, with another factor 2 for the spread of the gains: 100 e.
  * Any spectrum: a change in a direction that the matrix lacks grows by
    3.4445^5 = 485 while the iterate ends at norm ~ 1 or more: 5 C 485 e = 24000 e
    of the input's norm, one.
e is 2^-21 + sqrt(K) 2^-24 for fp32 (operands split into two fp16 of together 22
bits, half a step 2^-22 each, fp32 accumulation over K <= max(m, n) terms) and
2^-11 + 2^-11 for bf16 (both operands rounded to fp16), where the result's
rounding adds 2^-8.
"""
import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as mo
from paper_2404_11068_amd import graph as gr
from paper_2404_11068_amd import optim as op
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu


def _eps(dtype, m, n):
    return 2.0 ** -21 + math.sqrt(max(m, n)) * 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -10


def _check(got, ref, dtype, flat=True, name=""):
    got = to_f64(got)
    assert np.isfinite(got).all(), name
    for g, r in zip(got.reshape((-1,) + got.shape[-2:]), ref.reshape((-1,) + ref.shape[-2:])):
        e, size = _eps(dtype, *r.shape), np.linalg.norm(r)
        bound = 100 * e * size if flat else 24000 * e
        bound += (2.0 ** -8 if dtype == torch.bfloat16 else 0.0) * size
        assert np.linalg.norm(g - r) <= bound, (name, np.linalg.norm(g - r), bound)


SHAPES = [(1, 1), (1, 7), (5, 1), (2, 3), (16, 16), (17, 33), (31, 32), (32, 31), (64, 64), (23, 256), (256, 23),
          (128, 128), (65, 130), (130, 65), (128, 160), (129, 129), (127, 300), (256, 256), (300, 200), (192, 640),
          (1024, 96), (8, 2000), (385, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_flat_spectrum(m, n, dtype):
    print("\n[case] orthogonalize", m, n, dtype, flush=True)
    rng = np.random.default_rng(m * 1000 + n)
    # random signs and sizes on an orthonormal frame: singular values 0.5 .. 1, times 1e-3
    r = min(m, n)
    u = np.linalg.qr(rng.standard_normal((m, r)))[0] * rng.uniform(0.5, 1.0, r)
    x = torch.from_numpy(1e-3 * u @ np.linalg.qr(rng.standard_normal((n, r)))[0].T).to(dtype).cuda()
    got = op.orthogonalize(x)
    again = op.orthogonalize(x)
    assert got.dtype == dtype and torch.equal(got, again)
    _check(got, mo.orthogonalize(to_f64(x)), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,m,n", [(1, 40, 40), (5, 128, 128), (3, 200, 70), (2, 33, 500), (4, 256, 257), (40, 9, 12),
                                   # many enough to be taken a workgroup each, wide and tall, odd, up to 256 rows
                                   (78, 130, 200), (73, 256, 256), (72, 256, 290), (75, 250, 161), (74, 100, 700), (80, 520, 120),
                                   (72, 33, 1300), (72, 225, 585)])
def test_stacks(N, m, n, dtype):
    print("\n[case] stack", N, m, n, dtype, flush=True)
    rng = np.random.default_rng(N)
    x = torch.from_numpy(rng.standard_normal((N, m, n)) * 10.0 ** rng.integers(-6, 6, (N, 1, 1))).to(dtype).cuda()
    got = op.orthogonalize(x)
    _check(got, mo.orthogonalize(to_f64(x)), dtype, flat=False)
    for k in range(N):   # a matrix does not depend on its neighbours
        other = torch.randn_like(x)
        other[k] = x[k]
        assert torch.equal(got[k], op.orthogonalize(other)[k]), k
    y = x.clone()
    assert op.orthogonalize(y, out=y) is y and torch.equal(y, got)


@pytest.mark.parametrize("r,c", [(32, 1216), (64, 576), (96, 352), (128, 224), (160, 170), (192, 192)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_most_that_a_workgroup_holds(r, c, dtype):
    """Sizes at which X and a triangle fill the LDS, one row less, and a unit more, wide and tall."""
    for m, n in ((r, c), (c, r - 1), (r, c + 1), (c, r + 1)):
        print("\n[case] orthogonalize", m, n, dtype, flush=True)
        x = torch.from_numpy(np.random.default_rng(m + n).standard_normal((2, m, n))).to(dtype).cuda()
        _check(op.orthogonalize(x), mo.orthogonalize(to_f64(x)), dtype, flat=False)


def _close(got, ref, dtype):
    """For any spectrum.  fp32: as _check.  bf16: all steps but the last two as fp32; a rounding of size 2^-11 in
    the last but one changes the iterate by C 2^-11 of its norm, which the last step's slope takes to 3.4445 times
    that and adds as much again: 10 (1 + 3.4445) 2^-11, and 2^-8 for the result's rounding."""
    got = to_f64(got)
    assert np.isfinite(got).all()
    for g, r in zip(got.reshape((-1,) + got.shape[-2:]), ref.reshape((-1,) + ref.shape[-2:])):
        size = np.linalg.norm(r)
        bound = 24000 * _eps(torch.float32, *r.shape)
        bound += (44.445 * 2.0 ** -11 + 2.0 ** -8) * size if dtype == torch.bfloat16 else 0.0
        assert np.linalg.norm(g - r) <= bound, (np.linalg.norm(g - r), bound)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,m,n", [
    # large tiles: up to 256 of them in a launch and more, fewer than eight matrices and more, wide and tall, odd
    (1, 1930, 2010), (1, 2100, 1990), (2, 1337, 1400), (13, 500, 530), (45, 300, 260), (24, 700, 390)])
def test_large_tiles(N, m, n, dtype):
    print("\n[case] large tiles", N, m, n, dtype, flush=True)
    x = torch.from_numpy(np.random.default_rng(N + m).standard_normal((N, m, n)).astype(np.float32)).to(dtype).cuda()
    got = op.orthogonalize(x)
    assert torch.equal(got, op.orthogonalize(x))
    k = N - 1
    _close(got[:1], mo.orthogonalize(to_f64(x[:1])), dtype)
    _close(got[k:], mo.orthogonalize(to_f64(x[k:])), dtype)
    other = torch.randn_like(x)
    other[k] = x[k]
    assert torch.equal(got[k], op.orthogonalize(other)[k])


@pytest.mark.parametrize("kind", ["gauss", "rank3", "decay"])
@pytest.mark.parametrize("N,m,n", [(1, 128, 128), (2, 60, 300), (1, 700, 300), (73, 200, 140), (75, 100, 700)])
def test_bf16_of_any_spectrum(kind, N, m, n):
    print("\n[case] bf16", kind, N, m, n, flush=True)
    rng = np.random.default_rng(17)
    x = rng.standard_normal((N, m, n))
    if kind == "rank3":
        x = rng.standard_normal((N, m, 3)) @ rng.standard_normal((N, 3, n))
    elif kind == "decay":
        u, s, v = np.linalg.svd(x, full_matrices=False)
        x = (u * np.exp(-np.arange(s.shape[1]) / s.shape[1] * 9)) @ v
    t = torch.from_numpy(x).to(torch.bfloat16).cuda()
    for steps in (1, 2, 3, 5, 7):
        _close(op.orthogonalize(t, steps=steps)[:2], mo.orthogonalize(to_f64(t[:2]), steps=steps), torch.bfloat16)


def test_muon_with_large_tiles():
    print("\n[case] muon, large tiles", flush=True)
    shapes = [(500, 530)] * 7 + [(530, 500)] * 6 + [(1, 1300), (300, 2), (777, 300)]
    rng = np.random.default_rng(4)
    P, G, M = ([rng.standard_normal(s).astype(np.float32) for s in shapes] for _ in range(3))
    gpu = lambda ts: [torch.from_numpy(t).cuda() for t in ts]
    p, g, m = gpu(P), gpu(G), gpu(M)
    opt = op.FusedMuonSWA(p, g, m, lr=0.1, adjust="none")
    opt.step()
    torch.cuda.synchronize()
    for k, s in enumerate(shapes):
        rp_, rm, rw = mo.muon_step(P[k], G[k], M[k], P[k], lr=0.1, momentum_decay=0.95, nesterov=True, weight_decay=0.0,
                                   swa_decay=0.999)
        e = 24000 * _eps(torch.float32, *s)
        assert np.linalg.norm(to_f64(m[k]) - rm) <= 2.0 ** -21 * (np.linalg.norm(M[k]) + np.linalg.norm(G[k])), s
        assert np.linalg.norm(to_f64(p[k]) - rp_) <= 0.1 * e + 2.0 ** -22 * np.linalg.norm(rp_), s
        assert np.linalg.norm(to_f64(opt.swa[k]) - rw) <= 0.1 * e + 2.0 ** -22 * np.linalg.norm(rw), s


@pytest.mark.parametrize("kind", ["rank1", "decay", "zero", "tiny", "huge", "one_entry"])
@pytest.mark.parametrize("m,n", [(96, 96), (150, 280)])
def test_hard_spectra(kind, m, n):
    print("\n[case] spectrum", kind, m, n, flush=True)
    rng = np.random.default_rng(7)
    x = rng.standard_normal((m, n))
    if kind == "rank1":
        x = np.outer(rng.standard_normal(m), rng.standard_normal(n))
    elif kind == "decay":
        u, s, v = np.linalg.svd(x, full_matrices=False)
        x = (u * np.exp(-np.arange(len(s)) / len(s) * 12)) @ v
    elif kind == "zero":
        x = x * 0
    elif kind == "one_entry":
        x = x * 0
        x[m // 2, n // 3] = -2.0
    x = x * {"tiny": 1e-30, "huge": 1e30}.get(kind, 1.0)
    for dtype in (torch.float32, torch.bfloat16):
        t = torch.from_numpy(x).to(dtype).cuda()
        eps = 1e-38 if kind == "tiny" else 1e-7
        _check(op.orthogonalize(t, eps=eps), mo.orthogonalize(to_f64(t), eps=eps), dtype, flat=False, name=kind)
    if kind == "zero":
        assert not op.orthogonalize(t).any()


def test_steps_coefs_and_eps():
    x = torch.from_numpy(np.random.default_rng(8).standard_normal((70, 90))).float().cuda()
    for steps, coefs in ((1, mo.COEFS), (2, mo.COEFS), (8, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))):
        _check(op.orthogonalize(x, steps=steps, coefs=coefs), mo.orthogonalize(to_f64(x), steps, coefs), torch.float32)
    # below eps the matrix is divided by eps: the steps see a norm of 1/2
    e = float(torch.linalg.vector_norm(x)) * 2
    _check(op.orthogonalize(x, eps=e), mo.orthogonalize(to_f64(x), eps=e), torch.float32)


def test_nan_and_infinity_stay_in_their_matrix():
    for m, n in ((40, 60), (200, 300)):
        x = torch.randn(3, m, n, device="cuda")
        want = op.orthogonalize(x)
        x[1, 3, 4] = float("nan")
        x[2, 0, 0] = float("inf")
        got = op.orthogonalize(x)
        assert got[1].isnan().all() and got[2].isnan().any() and torch.equal(got[0], want[0])


def test_memory_around_the_tensors_stays():
    for m, n in ((37, 53), (150, 131), (131, 150)):
        for dtype in (torch.float32, torch.bfloat16):
            for shift in (1, 2):
                k = 2 * m * n
                buf = torch.full((k + 300,), 9.0, dtype=dtype, device="cuda")
                x = torch.randn(2, m, n, device="cuda").to(dtype)
                src = torch.full((k + 300,), float("nan"), dtype=dtype, device="cuda")
                src[shift:shift + k] = x.reshape(-1)
                out = buf[shift:shift + k].view(2, m, n)
                op.orthogonalize(src[shift:shift + k].view(2, m, n), out=out)
                assert torch.equal(out, op.orthogonalize(x))
                assert (buf[:shift] == 9).all() and (buf[shift + k:] == 9).all()


LIST = [(128, 128), (256, 256), (4, 64), (1024, 256), (256, 1024), (23, 256), (50, 128), (518, 384), (1, 300), (37, 101),
        (300, 1), (0, 5), (128, 512), (65, 1), (129, 128)]


def _data(shapes, seed):
    rng = np.random.default_rng(seed)
    f = lambda scale: [(rng.standard_normal(s) * scale).astype(np.float32) for s in shapes]
    return dict(params=f(0.02), grads=f(1e-3), momentum=f(1e-4), swa=f(0.02))


def _flat(lists, shift=0):
    """The lists as views of one flat buffer each, `shift` elements into it."""
    out = []
    for arrays in lists:
        buf = torch.full((sum(a.size for a in arrays) + 2 * shift + 1,), 3.0, device="cuda")
        views, at = [], shift
        for a in arrays:
            v = buf[at:at + a.size].view(a.shape)
            v.copy_(torch.from_numpy(a))
            views.append(v)
            at += a.size
        out.append((buf, views))
    return out


@pytest.mark.parametrize("shapes,nesterov,wd,adjust,gscale,shift", [
    (LIST, True, 0.1, "spectral", None, 0),
    (LIST[::-1], False, 0.0, "rms", 0.25, 1),
    (LIST[:1], True, 0.0, "none", None, 2),
    ([(64, 64)] * 70, True, 0.01, "spectral", 2.0, 0),
    ([(200, 220)] * 3, False, 0.01, "spectral", None, 3),
    ([(200, 130)] * 190 + [(70, 520)] * 30 + [(600, 90)] * 9 + [(256, 200)] * 20, True, 0.01, "rms", 0.5, 1),
])
def test_muon_step(shapes, nesterov, wd, adjust, gscale, shift):
    """Three steps.  Bounds per element: fp32 roundings of the parameter (a few
    2^-24 of its largest value per step), and the update's error above times lr."""
    print("\n[case] muon", len(shapes), nesterov, wd, adjust, gscale, shift, flush=True)
    d = _data(shapes, 5)
    (pb, P), (gb, G), (mb, M), (wb, S) = _flat([d["params"], d["grads"], d["momentum"], d["swa"]], shift)
    opt = op.FusedMuonSWA(P, G, M, S, lr=0.02, momentum_decay=0.9, nesterov=nesterov, weight_decay=wd, swa_decay=0.9,
                          adjust=adjust)
    gs = None if gscale is None else torch.tensor([gscale], device="cuda")
    p, m, w = ([a.astype(np.float64) for a in d[k]] for k in ("params", "momentum", "swa"))
    grads = [torch.equal(g, torch.from_numpy(a).cuda()) for g, a in zip(G, d["grads"])]
    for _ in range(3):
        opt.step(grad_scale=gs)
        for i, (r, c) in enumerate(shapes):
            if r * c == 0:
                continue
            f = {"none": 1.0, "spectral": math.sqrt(max(1, r / c)), "rms": 0.2 * math.sqrt(max(r, c))}[adjust]
            p[i], m[i], w[i] = mo.muon_step(p[i], d["grads"][i], m[i], w[i], lr=0.02, momentum_decay=0.9,
                                            nesterov=nesterov, weight_decay=wd, swa_decay=0.9, update_scale=f,
                                            grad_scale=gscale or 1.0)
    torch.cuda.synchronize()
    for i, (r, c) in enumerate(shapes):
        if r * c == 0:
            continue
        f = {"none": 1.0, "spectral": math.sqrt(max(1, r / c)), "rms": 0.2 * math.sqrt(max(r, c))}[adjust]
        off = 3 * 0.02 * f * 24000 * _eps(torch.float32, r, c)
        size = math.sqrt(r * c) * 2.0 ** -24
        for got, ref, extra in ((P[i], p[i], off), (M[i], m[i], 0.0), (S[i], w[i], off)):
            bound = extra + 24 * size * max(np.abs(ref).max(), 0.1 * f if extra else 0.0)
            assert np.linalg.norm(to_f64(got) - ref) <= bound, (i, r, c)
    assert all(grads)
    for buf in (pb, gb, mb, wb):
        assert (buf[:shift] == 3).all() and (buf[buf.numel() - shift - 1:] == 3).all()


def test_muon_step_matches_orthogonalize_exactly_enough():
    """One step from zero momentum and parameters is -lr times the orthogonalised
    gradient: the two entry points agree to the fp32 bound of each."""
    for r, c in ((128, 128), (140, 260)):
        g = torch.randn(r, c, device="cuda")
        p = torch.zeros(r, c, device="cuda")
        opt = op.FusedMuonSWA([p], [g], lr=1.0, adjust="none", momentum_decay=0.95)
        opt.step()
        o = op.orthogonalize(g)
        assert torch.linalg.vector_norm(p + o) <= 2 * 24000 * _eps(torch.float32, r, c)


def test_muon_without_swa_and_repeatable():
    shapes = [(96, 200), (256, 256), (33, 7)]
    outs = []
    for k in range(2):
        d = _data(shapes, 9)
        P, G, M, S = ([torch.from_numpy(a).cuda() for a in d[n]] for n in ("params", "grads", "momentum", "swa"))
        tab = np.zeros(3, dtype=np.dtype(op.evo_muon_tensor))
        opt = op.FusedMuonSWA(P, G, M, S)
        if k:
            lib = op._muon_lib()
            for i, (p, g, m) in enumerate(zip(P, G, M)):
                tab[i] = (p.data_ptr(), g.data_ptr(), m.data_ptr(), 0, *p.shape, math.sqrt(max(1, p.shape[0] / p.shape[1])))
            assert lib.evo_muon_build_plan(tab.ctypes.data, 3, opt.plan.ctypes.data, opt.plan.nbytes) == 0
            opt.plan_device.copy_(torch.from_numpy(opt.plan))
        before = [s.clone() for s in S]
        opt.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) == bool(k) for a, b in zip(before, S))
        outs.append(P + M)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_muon_captured_replays():
    shapes = [(256, 256), (128, 128), (8, 128), (130, 300)]
    d = _data(shapes, 10)
    make = lambda: [[torch.from_numpy(a).cuda() for a in d[k]] for k in ("params", "grads", "momentum", "swa")]
    A, B = make(), make()
    one, two = op.FusedMuonSWA(*A, weight_decay=0.01), op.FusedMuonSWA(*B, weight_decay=0.01)
    scale = torch.ones(1, device="cuda")
    s = torch.cuda.Stream()
    cache = gr.GraphCache(capacity=1)
    for it in range(4):
        scale.fill_(0.5 + it)
        for g, h in zip(A[1], B[1]):
            g.normal_()
            h.copy_(g)
        torch.cuda.synchronize()
        one.step(grad_scale=scale)
        torch.cuda.synchronize()
        cache.run(1, lambda st: two.step(grad_scale=scale, stream=st), s)
        torch.cuda.synchronize()
        for x, y in zip(A[0] + A[2] + A[3], B[0] + B[2] + B[3]):
            assert torch.equal(x, y), it
        _ = torch.randn(1000, device="cuda").sum()


def test_orthogonalize_on_another_stream_and_in_a_graph():
    x = torch.randn(2, 140, 150, device="cuda")
    want = op.orthogonalize(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = op.orthogonalize(x, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    ws = torch.empty(op.orthogonalize_workspace_size(x.shape, x.dtype), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    cache = gr.GraphCache(capacity=1)
    for it in range(3):
        x.normal_()
        want = op.orthogonalize(x)
        ws.fill_(255)
        torch.cuda.synchronize()
        cache.run(1, lambda st: op.orthogonalize(x, out=out, workspace=ws, stream=st), s)
        torch.cuda.synchronize()
        assert torch.equal(out, want), it


def test_muon_refuses_tensors_that_overlap():
    """What a step writes may not be another matrix's (or its own) operand; gradients may be shared."""
    flat = torch.zeros(64 * 64, device="cuda")
    p, q, g = flat[:1024].view(32, 32), flat[1024:2048].view(32, 32), torch.randn(32, 32, device="cuda")
    op.FusedMuonSWA([p, q], [g, g]).step()                                       # neighbours, one gradient
    torch.cuda.synchronize()
    for params, grads, kw in (([p, p], [g, g], {}), ([p, flat[512:1536].view(32, 32)], [g, g], {}), ([p], [p], {}),
                              ([p], [flat[992:2016].view(32, 32)], {}), ([p], [g], dict(momentum=[p])),
                              ([p, q], [g, g], dict(swa=[q, p])), ([p], [g], dict(momentum=[q], swa=[q])),
                              ([p], [q], dict(momentum=[q]))):
        with pytest.raises(ValueError, match="overlap"):
            op.FusedMuonSWA(params, grads, **kw)
