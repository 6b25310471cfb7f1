"""Host-side checks of the attention to states of another length (no GPU): which tensors of a call may lie in one buffer.
Fake addresses, never touched; a workspace that is missing (status 4) shows that a call goes on."""
import pytest

from tests.test_cross_abi_host import A, BWD, FWD, _bwd, _dims, _fwd

PLAIN = dict(gate=None, bias=None, mask=None, dgate=None, dbias=None, ws=None)


def _packed(**kw):
    """Queries of 512 and keys of 128 channels in tokens of 1024 and 512."""
    d = dict(q_stride_row=10 * 1024, q_stride_tok=1024, k_stride_row=300 * 512, k_stride_tok=512)
    d.update(kw)
    return _dims(**d)


@pytest.mark.parametrize("shift,status", [(1024, 4), (-1024, 4), (512, 1), (-512, 1), (1008, 1), (1040, 1), (16, 1), (0, 1),
                                          (1024 + 2048, 4), (1024 + 5 * 2048, 4), (512 + 2048, 1)])
def test_packed_gradients_of_queries_and_gate(shift, status):
    # dgate beside dq in each token, or half under it
    assert _bwd(_packed(), dgate=A(11) + shift, ws=None) == status


@pytest.mark.parametrize("shift,status", [(256, 4), (512, 4), (768, 4), (128, 1), (240, 1), (800, 1), (1024, 1), (1280, 4)])
def test_packed_gradients_of_keys_and_values(shift, status):
    kw = dict(PLAIN, dv=A(12) + shift)
    assert _bwd(_packed(), **kw) == status


def test_gradients_of_queries_and_keys_in_one_buffer():
    # self-attention's projections: queries, keys and values of one token side by side
    d = dict(len_k=10, k_stride_row=10 * 1024, k_stride_tok=1024)
    for dk, dv, status in ((1024, 1280, 4), (1024, 1024, 1), (1024, 1264, 1), (1008, 1280, 1), (1024, 1808, 1), (1792, 1024, 4)):
        assert _bwd(_packed(**d), **dict(PLAIN, dk=A(11) + dk, dv=A(11) + dv)) == status, (dk, dv)


@pytest.mark.parametrize("rows", [1, 4])
def test_one_token_a_row(rows):
    """The token stride of a single token says nothing: blocks lie side by side within the row stride."""
    q = dict(n_rows=rows, rows_per_bias=1, len_q=1, q_stride_row=1024, o_stride_row=512)
    for tok in (512, 1024, 0):
        for shift, status in ((1024, 4), (512, 1), (1008, 1), (1536, 1 if rows > 1 else 4)):
            assert _bwd(_dims(**q, q_stride_tok=tok), dgate=A(11) + shift, ws=None) == status, (tok, shift)
    k = dict(n_rows=rows, rows_per_bias=1, len_k=1, k_stride_row=256)
    for tok in (128, 256):
        for shift, status in ((256, 4), (128, 1), (384, 1 if rows > 1 else 4)):
            assert _bwd(_dims(**k, k_stride_tok=tok), dv=A(12) + shift, ws=None) == status, (tok, shift)


def test_output_beside_the_queries():
    """The forward's output in another place of the tokens its queries lie in."""
    d = dict(len_q=10, len_k=3000, k_stride_row=384000, q_stride_row=10240, q_stride_tok=1024, o_stride_row=10240, o_stride_tok=1024)
    for shift, status in ((1024, 4), (1008, 1), (0, 1), (512, 1)):
        assert _fwd(_dims(**d), out=A(1) + shift, gate=None, ws=None) == status


def test_outputs_on_masks_statistics_and_workspaces():
    """Everything a call writes is apart from everything it reads or writes besides."""
    d = _dims(len_q=1, len_k=3000, q_stride_row=512, k_stride_row=384000, o_stride_row=512, rows_per_bias=1)
    assert _fwd(d, ws=None) == 4                                              # as it is, a call that lacks a workspace only
    for kw in (dict(out=FWD["bias"]), dict(out=FWD["mask"]), dict(out=FWD["lse"]), dict(out=FWD["lse"] - 4096 + 16),
               dict(lse=FWD["q"] + 64), dict(lse=FWD["gate"]), dict(lse=FWD["k"] + 4), dict(lse=FWD["v"]), dict(lse=FWD["bias"]),
               dict(lse=FWD["mask"] + 11996)):
        assert _fwd(d, **dict(kw, ws=None)) == 1, kw
    for name in ("q", "k", "v", "gate", "bias", "mask", "out", "lse"):
        assert _fwd(d, ws=FWD[name]) == 1 and _fwd(d, ws=FWD[name], ws_bytes=16) == 4, name
    assert _bwd(d, ws=None) == 4
    for out in ("dq", "dk", "dv", "dgate", "dbias"):
        for other in ("lse", "mask"):
            assert _bwd(d, **{out: BWD[other], "ws": None}) == 1, (out, other)
    for name in ("q", "k", "v", "gate", "bias", "mask", "out", "lse", "dout", "dq", "dk", "dv", "dgate", "dbias"):
        assert _bwd(d, ws=BWD[name]) == 1, name
