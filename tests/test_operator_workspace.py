"""The gradient's workspace holds a piece of the vocabulary for all tokens of at most the bytes that the header names, beside a few
values per token (no GPU needed)."""
import ctypes

import pytest

from paper_2411_17866_gb300 import dsm
from test_operator_args import ce, lib  # noqa: F401

VOCAB, WIDTH = 50257, 8


def up(v, to):
    return (v + to - 1) // to * to


@pytest.mark.parametrize("dtype,piece", [(dsm.BF16, 256 << 20), (dsm.F32, 512 << 20)])
@pytest.mark.parametrize("tokens", [39937, 60000, 70001, 100096, 131073, 333333, 500224])
def test_piece_of_the_vocabulary_is_bounded(lib, tokens, dtype, piece):  # noqa: F811
    pair = dtype == dsm.F32
    a = ce(dtype=dtype, tokens=tokens, vocab=VOCAB, width=WIDTH, h_stride=WIDTH, w_stride=WIDTH, w=4096)
    rows = up(tokens, 256)
    # per token: h (f32: as two pairs), the sums for dh, a few whole numbers; f32: W as a pair
    beside = rows * (2 * WIDTH * (4 if pair else 1) + 4 * 32 + 24) + pair * up(VOCAB, 256) * (4 * WIDTH + 4) + (1 << 16)
    least = 256 * rows * (8 if pair else 2)   # one piece of 256 rows of W, whatever it takes
    assert lib.dsm_linear_cross_entropy_workspace(ctypes.byref(a), 1) <= max(piece, least) + beside
