"""Host-side checks of the rotary positions (no GPU): which tensors of a call may lie in one buffer.  Fake addresses, never
touched; a workspace that is missing (status 4) shows that a call goes on."""
import pytest

from tests.test_rope_abi_host import FAKE, _bwd, _dims

AT = FAKE + (64 << 28)  # nothing else near


def _run(lens, heads, row, tok, dx0, dx1, rows=2):
    """dx0 and dx1 (bytes from AT) of packed strides (elements of bf16), everything else apart."""
    pair = lambda x: x if isinstance(x, tuple) else (x, x)
    d = _dims(n_rows=rows, len=lens, n_heads=heads, x_stride_row=pair(row), x_stride_tok=pair(tok),
              y_stride_row=tuple(l * h * 64 for l, h in zip(lens, heads)), y_stride_tok=tuple(64 * h for h in heads))
    far = FAKE + (128 << 28)
    return _bwd(d, dx0=AT + dx0, dx1=AT + dx1, x0=far, x1=far + (1 << 28), ws=None)


def test_rows_that_start_anywhere():
    """Tokens of 1280 bytes: 1024 of set 0, 256 of set 1; rows of half a token more than eight of them."""
    row = 8 * 640 + 320
    assert _run((4, 8), (8, 2), row, 640, 0, 1024) == 4
    assert _run((4, 6), (8, 2), row, 640, 0, 1024 + 2 * 1280) == 4     # its last tokens lie behind row 0, before row 1
    assert _run((4, 6), (8, 2), row, 640, 0, 1024 + 5 * 1280) == 1     # its row 0 reaches into row 1 of set 0
    assert _run((8, 8), (8, 2), row, 640, 0, 1024) == 4
    assert _run((8, 8), (8, 2), row, 640, 0, 1008) == 1


def test_rows_within_tokens():
    """Rows innermost: 1280 bytes each, tokens of two rows."""
    assert _run((4, 4), (8, 2), 640, 1280, 0, 1024) == 4
    assert _run((4, 4), (8, 2), 640, 1280, 0, 1664) == 1               # set 0's second row lies there
    assert _run((4, 4), (8, 2), 640, 1280, 0, 1024 + 2560) == 4


@pytest.mark.parametrize("tok", [(512, 128), (640, 640), (1024, 128)])
def test_one_token_a_row(tok):
    """The token stride of a single token says nothing: blocks lie side by side within the row stride."""
    for rows in (1, 2, 4):
        assert _run((1, 1), (8, 2), 640, tok, 0, 1024, rows) == 4
        assert _run((1, 1), (8, 2), 640, tok, 0, 1008, rows) == 1
        assert _run((1, 1), (8, 2), 640, tok, 0, 1040, rows) == (1 if rows > 1 else 4)
        assert _run((1, 1), (2, 8), 640, tok[::-1], 0, 256, rows) == 4
        assert _run((1, 1), (2, 8), 640, tok[::-1], 256 + 1024 - 16, 256, rows) == 1


def test_lengths_of_their_own_in_one_buffer():
    """One row of the batch, whose row stride says nothing either, and the last tokens' queries beside all keys."""
    assert _run((3, 16), (8, 2), (3 * 640, 16 * 640), 640, 13 * 1280, 1024, 1) == 4
    assert _run((3, 16), (8, 2), (3 * 640, 16 * 640), 640, 13 * 1280 + 16, 1024, 1) == 1
    assert _run((1, 16), (8, 2), (640, 16 * 640), (512, 640), 15 * 1280, 1024, 1) == 4
    assert _run((1, 16), (8, 2), 16 * 640, (512, 640), 15 * 1280, 1024, 3) == 4
    assert _run((1, 16), (8, 2), 16 * 640, (512, 640), 15 * 1280 - 16, 1024, 3) == 1


def test_gradients_beside_their_inputs():
    """dx in another place of the tokens x lies in, or dy."""
    d = _dims(n_rows=2, len=(16, 16), x_stride_row=(16 * 1024, 16 * 256), x_stride_tok=(1024, 256), y_stride_row=(16 * 512, 16 * 128))
    assert _bwd(d, x0=AT, dx0=AT + 1024, x1=AT + (1 << 28), dx1=AT + (1 << 28) + 256, ws=None) == 4
    assert _bwd(d, x0=AT, dx0=AT + 1008, x1=AT + (1 << 28), dx1=AT + (1 << 28) + 256, ws=None) == 1
