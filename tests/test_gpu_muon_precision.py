"""How near the Newton-Schulz results are to the fp64 oracle where the other
tests' bounds are wide: every form that a call can take (`FORMS`), both types,
ends of the coefficients' range, norms far below eps, rows far smaller than
others.

Tolerances, with e = 2^-21 + sqrt(K) 2^-24 (operands of 22 bits, half a step 2^-22 each,
fp32 accumulation over K <= max(m, n) terms).  A step's roundings change the
iterate by at most C e of itself, C = 10 (|a| + 2 |b| |A| + 4 |c| |A|^2) / gain, and where the
spectrum is flat the iterate grows along with the change: the changes of the steps add up,
and twice that for the spread of the gains, see `_flat`.  bf16 matrices go
through the same steps: their results are the fp32 ones of the same
values, rounded once, bit for bit.
"""
import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as mo
from paper_2404_11068_amd import optim as op
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu

# matrices, rows, columns: in LDS; a workgroup each, of up to 128 rows and of up to 256; tiles of 64 x 64; of 128 x 128
FORMS = [(1, 64, 64), (2, 352, 96), (3, 33, 7), (75, 100, 700), (73, 250, 161), (72, 256, 256), (1, 300, 260), (5, 200, 640),
         (1, 1930, 2010), (45, 300, 260)]
IDS = lambda f: "%dx%dx%d" % f


def _e(m, n):
    return 2.0 ** -21 + math.sqrt(max(m, n)) * 2.0 ** -24


def _frames(rng, N, m, n):
    """Matrices of singular values 0.5 .. 1, the first and the last of them different from the rest."""
    r = min(m, n)
    x = np.empty((N, m, n))
    some = [(np.linalg.qr(rng.standard_normal((m, r)))[0], np.linalg.qr(rng.standard_normal((n, r)))[0]) for _ in range(min(N, 3))]
    for k in range(N):
        u, v = some[0 if k == 0 else 2 if k == N - 1 and N > 2 else min(1, len(some) - 1)]
        x[k] = (u * rng.uniform(0.5, 1.0, r)) @ v.T
    return x


def _norms(x):
    return np.linalg.norm(x.reshape(x.shape[0], -1), axis=1)


def _ends(x):
    """First and last matrix: what a stack's others hold is covered by the tests of stacks."""
    return x if x.shape[0] < 3 else x[[0, -1]]


BF16 = FORMS + [(2, 128, 224), (2, 576, 64), (2, 1216, 32), (78, 130, 200), (80, 520, 120), (1, 150, 280), (24, 700, 390), (1, 1, 7)]


@pytest.mark.parametrize("form", BF16, ids=IDS)
def test_bf16_is_the_fp32_result_rounded(form):
    print("\n[case] bf16", form, flush=True)
    N, m, n = form
    rng = np.random.default_rng(1)
    kinds = [rng.standard_normal((N, m, n)), np.einsum("km,kn->kmn", *(rng.standard_normal((N, s)) for s in (m, n)))]
    kinds.append(kinds[0] * np.exp(-9 * rng.random((N, m, 1))) * 1e-20)
    for x in kinds:
        t = torch.from_numpy(x).to(torch.bfloat16).cuda()
        for steps in (1, 2, 3, 5, 8):
            got, full = (op.orthogonalize(v, steps=steps, eps=1e-30) for v in (t, t.float()))
            assert full.any() and torch.equal(got, full.to(torch.bfloat16)), steps


# coefficients that take singular values to 8 and hold them there (and a set that comes within 3e-4 of it once):
# entries of A = X X^T reach 64
AT_THE_END = [((1.5, -1 / 128, 0.0), 20), ((1.875, -1.25 / 64, 0.375 / 4096), 16)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_coefficients_at_the_end_of_their_range(form, dtype):
    """Slopes are at most the gains here, so changes add up: 2 steps C e of the result, C <= 10 (1.875 + 2.5 + 1.5)
    with |A| = 64 and gains of one and more."""
    print("\n[case] range", form, dtype, flush=True)
    N, m, n = form
    x = torch.from_numpy(_frames(np.random.default_rng(2), N, m, n)).to(dtype).cuda()
    for coefs, steps in AT_THE_END:
        got, ref = _ends(op.orthogonalize(x, steps=steps, coefs=coefs)), mo.orthogonalize(to_f64(_ends(x)), steps, coefs)
        assert np.abs(np.linalg.norm(ref, 2, (1, 2)) - 8).max() < 0.1
        bound = (2 * steps * 59 * _e(m, n) + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * _norms(ref)
        assert (_norms(to_f64(got) - ref) <= bound).all(), (_norms(to_f64(got) - ref), bound)


def test_one_singular_value_next_to_the_end():
    """2 s + b s^3 has its largest value, 7.99973, at s = 5.9998: a matrix of one entry that gets there in its fourth step.
    Each step's roundings, C = 10 (2 + 2 |b| 64) = 44 at most, are passed on by slopes of 2 at most: 2^8 44 e of 8."""
    top, steps = 5.9998, 8
    coefs = (2.0, -2 / (3 * top * top), 0.0)
    for m, n in ((5, 9), (40, 300), (200, 300)):
        lo, hi = 0.0, 1.0
        for _ in range(200):   # the start from which three steps lead to `top`
            mid = (lo + hi) / 2
            lo, hi = (mid, hi) if mo.singular_map(mid, 3, coefs) < top else (lo, mid)
        assert abs(mo.singular_map(hi, 4, coefs) - 2 * top / 1.5) < 1e-6 and hi < 1
        for dtype in (torch.float32, torch.bfloat16):
            x = torch.zeros(m, n, device="cuda")
            x[m // 2, n // 3] = hi
            x = x.to(dtype)
            for k in range(1, steps + 1):
                got, ref = to_f64(op.orthogonalize(x, steps=k, coefs=coefs, eps=1.0)), mo.orthogonalize(to_f64(x), k, coefs, 1.0)
                tol = 2 ** k * 44 * _e(m, n) * 8 + (2.0 ** -8 * np.abs(ref).max() if dtype == torch.bfloat16 else 0.0)
                assert np.abs(got - ref).max() <= tol, (m, n, dtype, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_norms_far_below_eps(form, dtype):
    """Divided by eps instead of the norm: singular values of norm / eps and less, flat: 2 steps C e of the result."""
    print("\n[case] below eps", form, dtype, flush=True)
    N, m, n = form
    x = _frames(np.random.default_rng(3), N, m, n)
    x = torch.from_numpy(x / _norms(x)[:, None, None] * 1e-9).to(dtype).cuda()
    for eps, steps in ((3e-9, 5), (1e-7, 5), (1e-4, 5), (1e-4, 8), (1e-1, 5), (1e1, 12), (1e16, 3)):
        got, ref = _ends(op.orthogonalize(x, eps=eps, steps=steps)), mo.orthogonalize(to_f64(_ends(x)), steps, eps=eps)
        bound = (2 * steps * 10 * _e(m, n) + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * _norms(ref)
        assert (_norms(to_f64(got) - ref) <= bound).all(), (eps, steps, _norms(to_f64(got) - ref), bound)


def test_muon_of_vanishing_gradients():
    """Momenta of norm 1e-13 at an eps of 1e-7, and zeros among them; the parameters are the update alone."""
    shapes = [(64, 64), (7, 33), (300, 260), (700, 90)] + [(200, 130)] * 80
    rng = np.random.default_rng(4)
    G = [_frames(rng, 1, *s)[0] * (0.0 if k % 9 == 5 else 20 * 1e-13 / math.sqrt(min(s))) for k, s in enumerate(shapes)]
    g = [torch.from_numpy(v.astype(np.float32)).cuda() for v in G]
    p = [torch.zeros_like(v) for v in g]
    op.FusedMuonSWA(p, g, lr=1.0, momentum_decay=0.95, nesterov=False, adjust="none").step()
    torch.cuda.synchronize()
    for k, s in enumerate(shapes):
        ref = -mo.orthogonalize(to_f64(g[k]) * 0.05)
        bound = (10 * 10 + 4) * _e(*s) * np.linalg.norm(ref)
        assert np.linalg.norm(to_f64(p[k]) - ref) <= bound, (k, s)


def _floor(X, steps):
    """What is added to a row of the iterate by the ends of fp16's range: X and A are held to 2^-40 per entry at the
    usual coefficients, P = a I + b A + c A A to 2^-39.  X's own error takes its entries' number in a row; P's and A's,
    which comes into P times |b| + 2 |c| |A|, 11 at most, are independent from entry to entry and go through P X, |X|_F.
    Each is passed on by slopes of 3.4445 at most.  X: the iterates."""
    own, made = math.sqrt(X[0].shape[1]) * 2.0 ** -40, 2.0 ** -39 + 11 * 2.0 ** -40
    return sum(3.4445 ** (steps - k) * own + 3.4445 ** (steps - k - 1) * made * np.linalg.norm(X[k]) for k in range(steps))


@pytest.mark.parametrize("ratio", [1e4, 1e6, 1e8])
@pytest.mark.parametrize("m,n", [(128, 224), (100, 700), (250, 300), (300, 250), (600, 800)])
def test_rows_far_larger_than_the_others(m, n, ratio):
    """Two rows of the short side are `ratio` times the others: the error of each row, and of the whole."""
    print("\n[case] rows", m, n, ratio, flush=True)
    rng = np.random.default_rng(5)
    for N in (1, 76) if max(m, n) < 800 and min(m, n) <= 256 else (1,):
        x = rng.standard_normal((N, min(m, n), max(m, n)))
        x[:, rng.choice(min(m, n), 2, replace=False)] *= ratio
        t = torch.from_numpy(x if m <= n else np.ascontiguousarray(x.swapaxes(1, 2))).float().cuda()
        one = to_f64(t[-1]) if m <= n else to_f64(t[-1]).T
        X = [one / np.linalg.norm(one)] + [mo.orthogonalize(one, k) for k in range(1, 13)]
        for steps in (5, 8, 12):
            got = to_f64(op.orthogonalize(t, steps=steps)[-1])
            off, rows = (np.linalg.norm(v, axis=1) for v in ((got if m <= n else got.T) - X[steps], X[steps]))
            e, floor = 20 * steps * _e(m, n), _floor(X, steps)
            assert (off <= e * rows + floor).all(), (N, steps, (off / (e * rows + floor)).max())
            assert np.linalg.norm(off) <= e * np.linalg.norm(rows) + floor * math.sqrt(min(m, n)), (N, steps)


def test_zeros_with_the_smallest_eps():
    for m, n in ((16, 24), (200, 300)):
        x = torch.zeros(2, m, n, device="cuda")
        x[1, 3, 4] = 1e-44
        for eps in (1e-300, 1e-306, 5e-324):
            got = op.orthogonalize(x, eps=eps)
            assert not got[0].any() and got[1].isfinite().all(), eps
            want = mo.singular_map(1.0)
            assert abs(float(got[1, 3, 4]) - want) <= 24000 * _e(m, n), eps


def _flat_tolerance(m, n, steps=5):
    return 20 * steps * _e(m, n)


@pytest.mark.parametrize("form", FORMS + [(76, 40, 600), (72, 256, 700), (1, 2100, 1990), (13, 500, 530)], ids=IDS)
def test_flat_spectra_in_every_form(form):
    """fp32's precision, not only that of any spectrum: changes add up over the steps."""
    print("\n[case] flat", form, flush=True)
    N, m, n = form
    x = torch.from_numpy(_frames(np.random.default_rng(6), N, m, n) * 1e-3).float().cuda()
    got, ref = _ends(op.orthogonalize(x)), mo.orthogonalize(to_f64(_ends(x)))
    off = _norms(to_f64(got) - ref)
    assert (off <= _flat_tolerance(m, n) * _norms(ref)).all(), off / _norms(ref)


@pytest.mark.parametrize("shapes", [
    [(64, 64), (90, 300), (7, 33), (1, 300), (300, 260), (650, 200)],                       # LDS and tiles of 64 x 64
    [(200, 130)] * 60 + [(70, 520)] * 30 + [(600, 90)] * 9 + [(256, 200)] * 20,             # a workgroup each
    [(500, 530)] * 7 + [(530, 500)] * 6 + [(777, 300)]], ids=["lds", "workgroups", "tiles128"])
def test_muon_of_flat_momenta(shapes):
    """The parameters' bound: the update's, the fp32 rounding of momentum and update (2^-22 of it), and two of the
    parameter, 2^-24 each.  The gradients are as they were afterwards."""
    print("\n[case] muon, flat", len(shapes), flush=True)
    rng = np.random.default_rng(7)
    G = [_frames(rng, 1, *s)[0].astype(np.float32) * 1e-2 for s in shapes]
    P = [(rng.standard_normal(s) * 0.02).astype(np.float32) for s in shapes]
    p, g = ([torch.from_numpy(v).cuda() for v in L] for L in (P, G))
    opt = op.FusedMuonSWA(p, g, lr=0.3, momentum_decay=0.9, weight_decay=0.1, swa_decay=0.75, adjust="rms")
    m, w = ([np.zeros(s) for s in shapes], P)
    w = [v.astype(np.float64) for v in P]
    q = [v.astype(np.float64) for v in P]
    for it in range(2):
        opt.step()
        torch.cuda.synchronize()
        for k, (r, c) in enumerate(shapes):
            f = 0.2 * math.sqrt(max(r, c))
            before = q[k]
            q[k], m[k], w[k] = mo.muon_step(before, G[k], m[k], w[k], lr=0.3, momentum_decay=0.9, nesterov=True,
                                            weight_decay=0.1, swa_decay=0.75, update_scale=f)
            update = np.linalg.norm(q[k] - 0.97 * before)
            bound = (it + 1) * (update * (_flat_tolerance(r, c) + 2.0 ** -21) + 2.0 ** -22 * np.linalg.norm(before))
            assert np.linalg.norm(to_f64(opt.momentum[k]) - m[k]) <= 2.0 ** -22 * (it + 1) * np.linalg.norm(m[k]), (it, k)
            assert np.linalg.norm(to_f64(p[k]) - q[k]) <= bound, (it, k, r, c)
            assert np.linalg.norm(to_f64(opt.swa[k]) - w[k]) <= bound + 2.0 ** -22 * np.linalg.norm(w[k]), (it, k, r, c)
    for a, b in zip(g, G):
        assert torch.equal(a.cpu(), torch.from_numpy(b))


@pytest.mark.parametrize("form", [f for f in FORMS if f[0] > 1] + [(3, 64, 64), (9, 500, 530)], ids=IDS)
def test_nan_and_infinity_in_every_form(form):
    """A NaN takes the whole of its matrix, and neither takes another one."""
    print("\n[case] nan", form, flush=True)
    N, m, n = form
    x = torch.randn(N, m, n, device="cuda")
    for eps in (1e-7, 1e9):
        want, y = op.orthogonalize(x, eps=eps), x.clone()
        y[0, m // 2, n - 1] = float("nan")
        y[N - 1, m - 1, 0] = float("-inf")
        got = op.orthogonalize(y, eps=eps)
        assert got[0].isnan().all() and got[N - 1].isnan().any(), eps
        assert torch.equal(got[1:N - 1], want[1:N - 1]), eps
        assert N < 3 or got[1:N - 1].isfinite().all()


def test_no_accepted_coefficients_leave_the_range():
    """Random coefficients and steps, refused or finite; inputs whose first singular values are one, and flat ones."""
    rng = np.random.default_rng(8)
    shapes = [(1, 40, 60), (73, 130, 150), (1, 150, 330)]
    inputs = []
    for N, m, n in shapes:
        one = np.zeros((N, m, n))
        one[:, m // 3, n // 2] = 1.0
        inputs += [torch.from_numpy(v).float().cuda() for v in (one, _frames(rng, N, m, n), rng.standard_normal((N, m, n)))]
    done = 0
    for _ in range(300):
        steps, coefs = int(rng.integers(1, 13)), (rng.uniform(-4, 5), rng.choice([0.0, rng.uniform(-8, 8)]), rng.choice([0.0, rng.uniform(-4, 4)]))
        if not op.orthogonalize_workspace_size((1, 40, 60), torch.float32, steps=steps, coefs=coefs):
            continue
        done += 1
        for eps in (1e-7, 1e3):
            assert all(op.orthogonalize(x, steps=steps, coefs=coefs, eps=eps).isfinite().all() for x in inputs), (steps, coefs, eps)
    assert done > 40
