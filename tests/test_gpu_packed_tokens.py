"""Packed buffers with one token a row of the batch, as single steps have them: views of them give the bits that tensors
of their own give, and what lies between stays."""
import pytest
import torch

from paper_2404_11068_amd import cross
from paper_2404_11068_amd import rope

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def _randn(seed, *shape, dtype):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


@DTYPES
@pytest.mark.parametrize("N,L", [(4, 1), (1, 1), (1, 7)])
def test_rotation_in_place(N, L, dtype):
    H, Hk, d = 8, 2, 64
    packed = _randn(1, N, L, H + 2 * Hk, d, dtype=dtype)
    before = packed.clone()
    q, k = packed[:, :, :H], packed[:, :, H:H + Hk]
    pos = torch.arange(100, 100 + L, dtype=torch.int32, device="cuda")
    steps, w = rope.rope_steps(rope.rope_frequencies(d)), torch.rand(d, device="cuda") + 0.5
    kw = dict(pos_k=pos, norm=True, weight_q=w, weight_k=w)
    want = rope.rope_fwd(q.contiguous(), pos, steps, k=k.contiguous(), **kw)
    dq, dk = _randn(2, N, L, H, d, dtype=dtype), _randn(3, N, L, Hk, d, dtype=dtype)
    gwant = rope.rope_bwd(dq, pos, steps, dk=dk, q=q.contiguous(), k=k.contiguous(), **kw)
    grads = torch.full_like(packed, 7.0)
    got = rope.rope_bwd(dq, pos, steps, dk=dk, q=q, k=k, out_q=grads[:, :, :H], out_k=grads[:, :, H:H + Hk], **kw)
    rope.rope_fwd(q, pos, steps, k=k, out_q=q, out_k=k, **kw)
    torch.cuda.synchronize()
    for a, b in zip(got, gwant):
        assert torch.equal(a, b)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(packed[:, :, H + Hk:], before[:, :, H + Hk:])
    assert (grads[:, :, H + Hk:] == 7.0).all()


@DTYPES
def test_last_queries_beside_all_keys(dtype):
    """One row: the queries of the last tokens in the buffer that holds the keys of all."""
    H, Hk, d, L = 4, 2, 32, 9
    packed = _randn(4, 1, L, H + Hk, d, dtype=dtype)
    q, k = packed[:, L - 2:, :H], packed[:, :, H:]
    pos = torch.arange(L, dtype=torch.int32, device="cuda")
    steps = rope.rope_steps(rope.rope_frequencies(d))
    want = rope.rope_fwd(q.contiguous(), pos[L - 2:].contiguous(), steps, k=k.contiguous(), pos_k=pos)
    rest = packed[:, :L - 2, :H].clone()
    rope.rope_fwd(q, pos[L - 2:].contiguous(), steps, k=k, pos_k=pos, out_q=q, out_k=k)
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(packed[:, :L - 2, :H], rest)


@DTYPES
@pytest.mark.parametrize("N,Lq,Lk", [(4, 1, 30), (4, 30, 1), (3, 1, 1)])
def test_gradients_of_single_tokens_in_packed_buffers(N, Lq, Lk, dtype):
    H, d = 4, 32
    qg, kv = _randn(5, N, Lq, 2 * H, d, dtype=dtype), _randn(6, N, Lk, 2 * H, d, dtype=dtype)
    q, g, k, v = qg[:, :, :H], qg[:, :, H:], kv[:, :, :H], kv[:, :, H:]
    c = [t.contiguous() for t in (q, k, v, g)]
    dout = _randn(7, N, Lq, H, d, dtype=dtype)
    out, lse = cross.cross_attn_fwd(*c)
    want = cross.cross_attn_bwd(*c, None, None, out, lse, dout)
    dqg, dkv = torch.full_like(qg, 7.0), torch.full_like(kv, 7.0)
    got = cross.cross_attn_bwd(q, k, v, g, None, None, out, lse, dout, dq=dqg[:, :, :H], dgate=dqg[:, :, H:], dk=dkv[:, :, :H],
                               dv=dkv[:, :, H:])
    torch.cuda.synchronize()
    for a, b in zip(got[:4], want[:4]):
        assert torch.equal(a, b)
