"""Vectors that do not start on their elements' boundaries are refused before any CUDA call (no GPU needed)."""
import ctypes

import pytest

from paper_2411_17866_gb300 import dsm
from test_operator_args import ce, lib  # noqa: F401


@pytest.mark.parametrize("offset", [1, 2, 3])
@pytest.mark.parametrize("tokens", [1, 10, 300])
@pytest.mark.parametrize("dtype", [dsm.BF16, dsm.F32])
def test_misaligned_vectors_are_refused(lib, dtype, tokens, offset):  # noqa: F811
    a, bad = ctypes.byref(ce(dtype=dtype, tokens=tokens)), 4096 + offset
    for loss, lse in ((bad, 8192), (8192, bad), (bad, bad)):
        assert lib.dsm_linear_cross_entropy(a, loss, lse, 4096, 1 << 40, None) == dsm.DSM_EALIGN
        assert "loss and lse" in dsm.last_error()
        assert lib.dsm_linear_cross_entropy_grad(a, loss, lse, 1, 4096, 64, 4096, 64, 4096, 1 << 40, None) == dsm.DSM_EALIGN
        assert "lse and grad_loss" in dsm.last_error()
