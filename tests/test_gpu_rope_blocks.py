"""GPU parity of rotary positions and norms of heads where a workgroup takes several tokens, up to 16 from 32768 tokens
on: rows that end inside its tokens, several rows of one to fifteen tokens in one of them, and strides of more than 2^24
elements.  The comparison with the oracle and its bounds are those of the smaller cases."""
import numpy as np
import pytest
import torch

from paper_2404_11068_amd import rope
from tests import test_gpu_rope as base

pytestmark = pytest.mark.gpu

CASES = [
    # N, Lq, Lk, H, Hk, d, rot, interleaved, far
    (40000, 1, 1, 1, 1, 16, 16, False, 100000),
    (40000, 1, 0, 3, 0, 8, 8, True, 0),
    (6000, 7, 3, 1, 2, 16, 12, False, -500),
    (6000, 7, 3, 2, 1, 24, 24, True, 0),
    (3500, 15, 2, 1, 1, 16, 16, False, 7),
    (1100, 15, 1, 2, 3, 40, 24, False, 0),
    (4100, 1, 1, 2, 1, 16, 8, False, 3),
    (3001, 3, 1, 1, 1, 32, 32, True, 2 ** 30),
    (2, 20011, 13003, 1, 1, 16, 16, False, 5),
    (3, 11003, 17, 2, 5, 16, 6, False, 0),
    (17, 2003, 1001, 1, 1, 24, 16, True, 0),
    (70, 19, 470, 1, 3, 8, 8, False, 0),
]


@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "N%d_%dx%d_H%d_%d_d%d_r%d_%s_%d" % c)
def test_several_tokens_a_workgroup(case, dtype, norm):
    base.test_forward_and_backward(case, dtype, norm)


@pytest.mark.parametrize("L", [5, 40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_far_strides(dtype, L):
    """Tokens 2^24 elements and more apart, rows within them, and rows so far apart: the bits of packed tensors."""
    N, H, d = 3, 2, 64
    far = (1 << 24) + 8 * 64 if L == 5 else 1 << 20
    rng = np.random.default_rng(61)
    q, dq = (base._rand(rng, (N, L, H, d), dtype) for _ in range(2))
    pos = torch.from_numpy(rng.integers(0, 1000, (N, L)).astype(np.int32)).cuda()
    steps, w = rope.rope_steps(rope.rope_frequencies(d)), torch.ones(d, device="cuda")
    room = torch.empty(far * max(L, N) + N * H * d, dtype=dtype, device="cuda")
    for strides in ((H * d, far, d, 1), (far, H * d, d, 1)):
        view = room.as_strided((N, L, H, d), strides)
        for norm in (False, True):
            kw = dict(norm=norm, weight_q=w if norm else None)
            want, _ = rope.rope_fwd(q, pos, steps, **kw)
            view.copy_(q)
            got, _ = rope.rope_fwd(view, pos, steps, **kw)
            rope.rope_fwd(view, pos, steps, out_q=view, **kw)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(view, want)
            if norm:
                view.copy_(q)
                want = rope.rope_bwd(dq, pos, steps, q=q, **kw)
                got = rope.rope_bwd(dq, pos, steps, q=view, out_q=view, **kw)
                torch.cuda.synchronize()
                assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
