"""GPU parity of the relative position bias where the other tests do not go:
edges that span more than 2^31, and onto a base with every number of heads that
share a lane's buckets.

Tolerances as in test_gpu_relpos: without a base the fp32 result is the
table's entry itself; sums of integers below 2^24 are exact; with a base one fp32
addition (2^-24 of the result) and one rounding to the result's type (bf16: 2^-8).
"""
import numpy as np
import pytest
import torch

from oracle import relpos_oracle as ro
from paper_2404_11068_amd import relpos as rp
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Li,Lj", [(70, 129), (2600, 2503)])   # the forward searches in short calls, and has a table in long ones
@pytest.mark.parametrize("edges", [(-2 ** 30 - 5, 0, 2 ** 30 + 5), (-2 ** 30 - 5, 0, 7, 2 ** 30 + 5),
                                   (-2 ** 31 + 3, -5 * 10 ** 8, -5, 10 ** 9, 2 ** 31 - 1)], ids=["three", "four", "ends"])
def test_edges_that_span_more_than_an_int(edges, Li, Lj):
    """At most one edge in a step of the table, whose first and last differences are more than 2^31 apart."""
    print("\n[case] wide edges", edges, Li, Lj, flush=True)
    rng = np.random.default_rng(3)
    edges, H = np.array(edges), 2
    pi, pj = rng.integers(-2 ** 31, 2 ** 31, Li), rng.integers(-2 ** 31, 2 ** 31, Lj)
    pi[:20], pj[:20] = rng.integers(-9, 9, 20), rng.integers(-9, 9, 20)
    pi[20:40], pj[20:40] = rng.choice(edges, 20), rng.choice([-1, 0, 1, 2 ** 31 - 1, -2 ** 31], 20)
    t = lambda a: torch.from_numpy(a.astype(np.int32)).cuda().view(1, -1)
    diff = np.clip(pi[:, None].astype(np.int64) - pj[None, :], -2 ** 31, 2 ** 31 - 1)
    n = np.searchsorted(edges, diff, side="right")
    table = torch.from_numpy(rng.standard_normal((H, len(edges) + 1)).astype(np.float32)).cuda()
    out = rp.relpos_bias_fwd(t(pi), t(pj), t(edges).view(-1), table, dtype=torch.float32)
    assert np.array_equal(out[0].cpu().numpy(), table.cpu().numpy()[:, n])
    g = rng.integers(-9, 10, (1, H, Li, Lj)).astype(np.float32)
    d = rp.relpos_bias_bwd(t(pi), t(pj), t(edges).view(-1), torch.from_numpy(g).cuda())
    assert np.array_equal(to_f64(d), np.stack([np.bincount(n.reshape(-1), g[0, h].reshape(-1), len(edges) + 1) for h in range(H)]))


def _heads_per_lane(B, H, Li, Lj):
    """The forward's rule: as many heads as there are, up to eight, while the groups' workgroups number 256."""
    wg = B * -(-(Li * -(-Lj // 8)) // 256)
    return next((n for n in (8, 4, 2) if H > n // 2 and wg * -(-H // n) >= 256), 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,H,Li,Lj,seg,heads", [
    (1, 8, 384, 384, False, 2), (1, 7, 383, 385, True, 2), (2, 3, 290, 450, True, 2),        # two, the last group short
    (1, 8, 512, 512, False, 4), (1, 6, 640, 511, True, 4), (3, 3, 413, 423, False, 4), (1, 11, 500, 509, True, 4),
    (1, 8, 768, 768, False, 8), (2, 5, 513, 517, True, 8), (1, 13, 700, 601, False, 8), (1, 16, 33000, 7, True, 8)])
def test_onto_a_base_with_several_heads_per_lane(B, H, Li, Lj, seg, heads, dtype):
    print("\n[case] heads", B, H, Li, Lj, seg, heads, dtype, flush=True)
    assert _heads_per_lane(B, H, Li, Lj) == heads
    rng = np.random.default_rng(H * Li)
    num = lambda lo, hi, *s: torch.from_numpy(rng.integers(lo, hi, s).astype(np.int32)).cuda()
    pi, pj = num(-80, 80, B, Li), num(-80, 80, B, Lj)
    si, sj = (num(0, 3, B, Li), num(0, 3, B, Lj)) if seg else (None, None)
    edges = rp.relpos_edges_log(16, 256)
    table = torch.from_numpy(rng.standard_normal((H, edges.numel() + 1 + seg)).astype(np.float32)).cuda()
    size = B * H * Li * Lj
    room = torch.full((size + 24,), 7.0, dtype=dtype, device="cuda")
    base = torch.from_numpy(rng.standard_normal((B, H, Li, Lj)).astype(np.float32)).cuda().to(dtype)
    base[0, 0, 0, 0], base[-1, -1, -1, -1] = float("-inf"), float("-inf")
    out = room[5:5 + size].view(B, H, Li, Lj)                       # rows aligned to their element, no more
    kw = dict(seg_i=si, seg_j=sj)
    rp.relpos_bias_fwd(pi, pj, edges, table, base=base, out=out, **kw)
    alone = rp.relpos_bias_fwd(pi, pj, edges, table, dtype=dtype, **kw)
    inplace = base.clone()
    rp.relpos_bias_fwd(pi, pj, edges, table, base=inplace, out=inplace, **kw)
    assert torch.equal(inplace, out) and (room[:5] == 7).all() and (room[5 + size:] == 7).all()
    index = [t if t is None else t.cpu().numpy() for t in (pi, pj, edges, table)]
    seg_ = [t if t is None else t.cpu().numpy() for t in (si, sj)]
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    ref = ro.forward(*index, None, *seg_)
    assert (np.abs(to_f64(alone) - ref) <= step * np.abs(ref)).all()
    ref, got = ref + to_f64(base), to_f64(out)
    assert got[0, 0, 0, 0] == got[-1, -1, -1, -1] == -np.inf
    fin = np.isfinite(ref)
    assert (np.abs(got[fin] - ref[fin]) <= (step * (1 + 2.0 ** -24) + 2.0 ** -24) * np.abs(ref[fin])).all()
