"""The operators on values that lie far from the ordinary: logits far below zero, rows and entries of very different sizes.

Losses are held to 1e-5 of the largest logit, gradients to the bounds of test_gpu_operators.check(), unless a test says
more.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2411_17866_gb300 import dsm  # noqa: E402
from test_gpu_operators import ce64, check, problem  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.manual_seed(5)


# ---- logits far below zero ----------------------------------------------------------------------------------------

def shifted(tokens, vocab, width, dtype, shift, rows=slice(None)):
    """problem() with the logits of some rows of W moved by `shift` (a multiple of 8, so that bf16 holds it)."""
    h, w, y, a = problem(tokens, vocab, width, dtype, lean=8.0)
    h[:, 0] = 8
    w[:, 0] = 0
    w[rows, 0] = shift / 8
    return h, w, y, a


def check_loss(h, w, y, a):
    """The loss by itself, and that the gradients are finite."""
    loss, lse = dsm.linear_cross_entropy(h, w, y)
    want = ce64(h, w, y, a)
    for got, ref in ((loss, want[0]), (lse, want[1])):
        assert bool(((got.double() - ref).abs() < 1e-5 * want[4]).all())
    assert all(bool(g.isfinite().all()) for g in dsm.linear_cross_entropy_grad(h, w, y, lse, a))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 3, 16, 100, 300])
@pytest.mark.parametrize("shift", [-56, -88, -96, -120, -400])
def test_all_logits_far_below_zero(shift, tokens, dtype):
    """A shift of all logits changes neither loss nor gradient: nothing may depend on where zero lies."""
    check_loss(*shifted(tokens, 1030, 96, dtype, shift))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 3, 16, 100, 300])
@pytest.mark.parametrize("first,last", [(0, 32), (0, 128), (128, 256), (32, 1030), (900, 1030), (512, 513)])
def test_some_logits_far_below_zero(first, last, tokens, dtype):
    """Whole groups of columns, at the start of a tile or behind its start, that add nothing to the others' sums."""
    check(*shifted(tokens, 1030, 96, dtype, -120, slice(first, last)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 60, 200])
def test_logits_far_below_zero_over_a_large_vocabulary(tokens, dtype):
    check_loss(*shifted(tokens, 50257, 64, dtype, -120))
    check_loss(*shifted(tokens, 50257, 64, dtype, -240, slice(7, 40000)))
