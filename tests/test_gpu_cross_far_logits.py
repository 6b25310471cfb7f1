"""GPU parity of the attention to states of another length where logits lie far
from zero: biases between ordinary values and the type's lowest, as masks are
made of, at some keys or at all keys of a query.

Bounds as in the parity tests of the ordinary range.  A logit is formed in fp32,
so that a far one keeps nothing of q k' unless it is a multiple of its step: here
queries and keys lie in different halves of the head, q k' is zero without any
rounding, and the logits are the biases.  Softmax and its gradients do not
change with a constant added to a query's logits, so the bounds are those at
biases less the query's largest where that is beyond a thousand (ordinary
ones keep the log-sum-exp's rounding in their bounds); the log-sum-exp itself is
an fp32 number (4 F of its size).
"""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paper_2404_11068_amd import cross
from tests.parity_util import to_f64
from tests.test_gpu_cross import F, _bounds, _check, _close, _draw

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
LOW = [-1e6, -1e8, -1e10, -1e15, -1e20, -0.9e30, -1.2e30, -1e35, "half"]
# N, Lq, Lk, H, Hk, d, copies: single tokens, tiles of queries, the keys split over workgroups, and rows of the batch walked
# over (as often as the last number says the same ones)
SHAPES = [(2, 1, 200, 4, 4, 32, 1), (2, 70, 200, 4, 2, 64, 1), (1, 40, 3000, 2, 2, 128, 1), (1, 1, 3000, 2, 1, 128, 1),
          (2, 130, 77, 4, 4, 32, 64), (2, 2, 50, 2, 2, 16, 1024)]
IDS = ["token", "rows", "rows_split", "token_split", "short", "short_one"]


def _value(low, dtype):
    return torch.finfo(dtype).min / 2 if low == "half" else low


def _apart(q, k):
    """Queries on the first half of the channels, keys on the second."""
    q[..., q.shape[3] // 2:] = 0
    k[..., :k.shape[3] // 2] = 0


def _far_bounds(f, mm, do, rpb, u):
    """Bounds at biases less each query's largest, where that is far."""
    q, k, v, g, bias = f
    x = bias if mm is None else np.where((mm == 0).all(0), -np.inf, bias)
    x = np.where(x > -1e30, x, -np.inf)
    top = x.max(-1, keepdims=True, initial=-np.inf)
    return _bounds(q, k, v, g, np.where(np.isfinite(top), x - np.where(np.abs(top) > 1000, top, 0.0), -np.inf), mm, do, rpb, u)


def _forward(q, k, v, g=None, bias=None, m=None, copies=1):
    """(out, lse) of the rows, run `copies` times over in one call, one bias for all: the copies are alike."""
    many = [None if t is None else t.repeat((copies,) + (1,) * (t.dim() - 1)) for t in (q, k, v, g)]
    out, lse = cross.cross_attn_fwd(*many, bias, None if m is None else m.repeat(copies, 1))
    torch.cuda.synchronize()
    both = []
    for t in (out, lse):
        t = t.view((copies, q.shape[0]) + t.shape[1:])
        assert bool((t[:1] == t).all() | (t != t).any()), "copies differ"
        both.append(t[0])
    return both


def _check_far(args, rpb=None, backward=True, copies=1):
    q, k, v, g, bias, m, dout = args
    u = 2.0 ** -8 if q.dtype == torch.bfloat16 else F
    f = [None if t is None else to_f64(t) for t in (q, k, v, g, bias)]
    mm, do = None if m is None else m.cpu().numpy().astype(np.uint8), to_f64(dout)
    assert rpb is None or copies == 1
    out, lse = _forward(q, k, v, g, bias, m, copies) if rpb is None else cross.cross_attn_fwd(q, k, v, g, bias, m, rows_per_bias=rpb)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref = co.forward(*f, mm, rpb)[:2]
        b = _far_bounds(f, mm, do, rpb or q.shape[0], u)
    _close(out, ref[0], b[0], u, "out")
    _close(lse, ref[1], b[1] + 4 * F * np.where(np.isfinite(ref[1]), np.abs(ref[1]), 0.0), 0.0, "lse")
    if backward:
        grads = cross.cross_attn_bwd(q, k, v, g, bias, m, out, lse, dout, rows_per_bias=rpb)
        torch.cuda.synchronize()
        with np.errstate(invalid="ignore"):
            want = co.backward(*f, mm, do, rpb)
        for name, got, r, bound in zip(("dq", "dk", "dv", "dgate", "dbias"), grads, want, b[2:]):
            assert (got is None) == (r is None), name
            if got is not None:
                _close(got, r, bound, u, name)


@DTYPES
@pytest.mark.parametrize("low", LOW)
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_far_keys_before_ordinary_ones(shape, low, dtype):
    """The first keys of every query (more than a step of them), or all but the last, at a bias far below the others'."""
    N, Lq, Lk, H, Hk, d, copies = shape
    args = _draw((N, Lq, Lk, H, Hk, d, False, 1, None), dtype, 21)
    bias = args[4]
    bias[:, 0, :, :min(Lk - 1, 130)] = _value(low, dtype)
    bias[:, 1, :, :Lk - 1] = _value(low, dtype)
    with np.errstate(invalid="ignore"):
        f = [None if t is None else to_f64(t) for t in args[:5]]
        ref, b = co.forward(*f)[:2], _bounds(*f, None, to_f64(args[6]), N, 2.0 ** -8 if dtype == torch.bfloat16 else F)
    out, lse = _forward(*args[:5], copies=copies)
    _close(out, ref[0], b[0], 2.0 ** -8 if dtype == torch.bfloat16 else F, "out")
    _close(lse, ref[1], b[1], 0.0, "lse")


@DTYPES
@pytest.mark.parametrize("low", LOW)
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_queries_with_far_keys_only(shape, low, dtype):
    """All keys of some queries far below: equally likely where they still are keys, none of them below -1e30."""
    N, Lq, Lk, H, Hk, d, copies = shape
    args = _draw((N, Lq, Lk, H, Hk, d, True, 1, None), dtype, 22)
    _apart(*args[:2])
    args[4][:, :, ::2] = _value(low, dtype)
    _check_far(args, backward=False, copies=copies)
    if dtype == torch.float32 and low != "half" and abs(low) < 1e20:
        # neighbouring numbers: each a step of fp32 from the next
        b = args[4][:, :, ::2]
        step = float(np.spacing(np.float32(abs(low))))
        b += step * torch.randint(-2, 3, b.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
        _check_far(args, backward=False, copies=copies)


@DTYPES
@pytest.mark.parametrize("shape", SHAPES[:4], ids=IDS[:4])
def test_far_keys_in_order(shape, dtype):
    """Biases that rise from the lowest to ordinary ones along the keys, and fall back, and logits far above zero."""
    N, Lq, Lk, H, Hk, d, copies = shape
    args = _draw((N, Lq, Lk, H, Hk, d, True, 1, "random"), dtype, 23)
    _apart(*args[:2])
    args[5][:] = args[5][:1]
    args[5][:, Lk // 2] = 1
    e = torch.linspace(0, 30, Lk, device="cuda")
    args[4][:, 0] = (-(10.0 ** (30 - e))).to(dtype)
    args[4][:, 1] = (10.0 ** e).to(dtype)
    if H > 2:
        args[4][:, 2] = (-(10.0 ** e)).to(dtype)
        args[4][:, 3] = torch.finfo(dtype).max
    _check_far(args, backward=False, copies=copies)


@DTYPES
def test_the_edge_of_no_key(dtype):
    """A natural logit of -1e30: the numbers next to it on both sides."""
    N, Lq, Lk, H, d = 2, 6, 90, 2, 32
    args = _draw((N, Lq, Lk, H, H, d, False, 1, None), dtype, 24)
    _apart(*args[:2])
    at = torch.tensor(-1e30, dtype=dtype, device="cuda")
    up, down = torch.nextafter(at, torch.zeros_like(at)), torch.nextafter(at, torch.full_like(at, -float("inf")))
    near = torch.stack([torch.nextafter(up, torch.zeros_like(at)), up, at, down, torch.nextafter(down, torch.full_like(at, -float("inf"))),
                        torch.tensor(-0.8e30, dtype=dtype, device="cuda")])
    args[4][:] = near.view(1, 1, Lq, 1)
    for copies, keys in ((1, Lk), (1024, 50)):
        some = args[:1] + tuple(t[:, :keys].contiguous() for t in args[1:3]) + (None, args[4][..., :keys].contiguous(), None, args[6])
        _check_far(some, backward=False, copies=copies)
    assert float(near[5]) > -1e30 > float(near[4])


def _same_keys(N, Lq, Lk, H, d, size, dtype, seed):
    """Queries and keys whose logits are all the same number of about `size`: one channel of each makes it, the others of
    the keys meet zeros."""
    args = _draw((N, Lq, Lk, H, H, d, False, 0, None), dtype, seed)
    q, k = args[:2]
    q[..., 0], q[..., 1:d // 2], q[..., d // 2:] = 1.0, 0.0, 1.0
    k[..., 0], k[..., d // 2:] = 1.0, 0.0
    root = float(np.sqrt(abs(size) * np.sqrt(d)))
    q[..., 0] *= torch.tensor(root, dtype=dtype, device="cuda") * (1 if size > 0 else -1)
    k[..., 0] *= torch.tensor(root, dtype=dtype, device="cuda")
    return args


@DTYPES
@pytest.mark.parametrize("size", [3e3, 1e6, -1e7, 1e10, -3e10, 1e15, -1.1e15])
@pytest.mark.parametrize("N,Lq,Lk,H,d,copies", [(2, 1, 301, 2, 64, 1), (2, 70, 301, 2, 32, 1), (1, 40, 3000, 1, 128, 1),
                                                (2, 130, 77, 4, 32, 64)], ids=["token", "rows", "split", "short"])
def test_far_products(N, Lq, Lk, H, d, copies, size, dtype):
    """Without a bias: the products of queries and keys alone are far from zero, and the same for all keys."""
    args = _same_keys(N, Lq, Lk, H, d, size, dtype, 25)
    q, k, v = args[:3]
    u = 2.0 ** -8 if dtype == torch.bfloat16 else F
    out, lse = _forward(q, k, v, copies=copies)
    f = [to_f64(t) for t in (q, k, v)]
    ref = co.forward(*f)
    f[0][..., 0] = 0.0
    b = _bounds(*f, None, None, None, to_f64(args[6]), N, u)
    _close(out, np.broadcast_to(f[2].mean(1, keepdims=True), out.shape), b[0], u, "out")
    _close(lse, ref[1], b[1] + 8 * F * np.abs(ref[1]), 0.0, "lse")
