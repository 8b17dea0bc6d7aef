"""Outputs inside wider rows, on 16-byte boundaries and with ends that are not: nothing beside them is written."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2411_17866_gb300 import dsm  # noqa: E402
from test_gpu_operators import TOL, check, orth64, problem, rel  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.manual_seed(5)


def inside(shape, row, dtype, offset=0):
    """A stack of matrices whose rows of shape[-1] lie `row` apart in a buffer of sevens, and a check that the rest stays so."""
    count, rows, cols = shape
    flat = torch.full((offset + count * rows * row + 64,), 7.0, dtype=dtype, device="cuda")
    out = flat[offset:offset + count * rows * row].view(count, rows, row)[:, :, :cols]
    rest = torch.ones_like(flat, dtype=torch.bool)
    rest[offset:offset + count * rows * row].view(count, rows, row)[:, :, :cols] = False
    return out, lambda: bool((flat[rest] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [3, 16, 50, 300])
@pytest.mark.parametrize("width", [1, 2, 3, 5, 7, 8, 9, 31, 33, 61, 64, 65, 127, 129, 250, 257])
def test_gradients_inside_wider_rows(width, tokens, dtype):
    h, w, y, a = problem(tokens, 300, width, dtype, 0.1)
    row = (width + 15) // 8 * 8
    (dh,), rest_h = inside((1, tokens, width), row, dtype)
    (dw,), rest_w = inside((1, 300, width), row, dtype)
    check(h, w, y, a, out_h=dh, out_weight=dw)
    assert rest_h() and rest_w()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", [(50, 1, 45), (4, 1, 45), (1, 300, 45), (1, 1, 3), (300, 1, 1), (50, 2, 301)])
def test_gradients_of_single_rows(tokens, vocab, width, dtype):
    """A single row has no row behind it whose boundary could say how far it may go."""
    h, w, y, a = problem(tokens, vocab, width, dtype)
    (dh,), rest_h = inside((1, tokens, width), width, dtype)
    (dw,), rest_w = inside((1, vocab, width), width, dtype)
    check(h, w, y, a, out_h=dh, out_weight=dw)
    assert rest_h() and rest_w()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 131, 163), (2, 300, 301), (2, 301, 150), (3, 400, 131), (13, 260, 279), (29, 131, 137),
                                   (24, 600, 1001), (24, 1001, 601), (40, 133, 139), (2, 60, 61), (2, 61, 60), (1, 1, 700), (1, 700, 1)])
def test_orthogonalized_matrices_inside_wider_rows(shape, dtype):
    g = torch.randn(shape, device="cuda").to(dtype)
    m = torch.zeros(shape, device="cuda")
    want = orth64(g)
    count, rows, cols = shape
    for row in ((cols + 15) // 8 * 8, cols):
        out, rest = inside(shape, row, dtype)
        dsm.orthogonalize(g, momentum=m.zero_(), mu=0.0, out=out)
        assert rel(out, want) < TOL[dtype] and rest()
    out, rest = inside((count, cols, rows), (rows + 15) // 8 * 8, dtype)
    gt = torch.empty(count, cols, rows, dtype=dtype, device="cuda").mT
    dsm.orthogonalize(gt.copy_(g), out=out.mT)
    assert rel(out.mT, want) < TOL[dtype] and rest()
    wide, rest = inside(shape, (cols + 15) // 8 * 8, dtype)
    wide.copy_(g)
    dsm.orthogonalize(wide, 0, out=wide)
    assert rel(wide, orth64(g, 0)) < 2.0 ** -8 and rest()
