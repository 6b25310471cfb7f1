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
