"""orthogonalize at sizes of all its tile shapes, both orientations, with ragged edges: every matrix of a stack by itself.

Tolerances are those of test_gpu_operators.py.  The tiles (CTAs per matrix instruction x columns) are chosen by
step_clocks() for the 152 SMs of a GB300; the comments say which ones that gives for bf16 and for f32.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2411_17866_gb300 import dsm  # noqa: E402
from test_gpu_operators import TOL, TOL_LOW_RANK, orth64  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [
    (24, 1000, 3000), (24, 3000, 1000), (24, 129, 4096), (6, 777, 1033),   # 2 x 256, 2 x 128
    (40, 133, 139), (40, 167, 131),                                        # 2 x 256, 1 x 128
    (39, 257, 515), (13, 260, 279), (20, 265, 131),                        # 1 x 128, 1 x 128
    (29, 131, 136), (27, 130, 129),                                        # 2 x 128, 2 x 128
    (1, 131, 163), (1, 138, 129), (2, 1100, 150),                          # 1 x 64, 1 x 64
]


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.manual_seed(5)


def worst(got, want):
    return float(((got.double() - want).norm(dim=(1, 2)) / want.norm(dim=(1, 2))).max())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_tiles(shape, dtype):
    g = torch.randn(shape, device="cuda").to(dtype)
    ws = dsm.orthogonalize_workspace(g)
    got = dsm.orthogonalize(g, workspace=ws)
    assert dsm.operator_status(ws) == 0
    assert worst(got, orth64(g)) < TOL[dtype]
    assert torch.equal(dsm.orthogonalize(g, workspace=ws), got)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_tiles_with_momentum_and_other_layouts(shape, dtype):
    """Rows off the 16-byte boundaries, and g and out transposed: the result leaves by plain stores."""
    count, rows, cols = shape
    g, m = torch.randn(shape, device="cuda").to(dtype), torch.randn(shape, device="cuda")
    want_m = 0.5 * m.double() + g.double()
    want = orth64(want_m)
    odd = torch.full((count, rows + 1, cols + 3), 7.0, dtype=dtype, device="cuda")
    out = odd[:, 1:, 2:-1]
    dsm.orthogonalize(g, momentum=m, mu=0.5, nesterov=False, out=out)
    assert worst(out, want) < TOL[dtype] and worst(m, want_m) < 2.0 ** -22
    edge = torch.ones_like(odd, dtype=torch.bool)
    edge[:, 1:, 2:-1] = False
    assert bool((odd[edge] == 7).all())
    turned = torch.empty(count, cols, rows, dtype=dtype, device="cuda").mT
    dsm.orthogonalize(want_m.float().to(dtype) if dtype == F32 else g, out=turned)
    assert worst(turned, want if dtype == F32 else orth64(g)) < TOL[dtype]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(24, 600, 1000), (24, 1000, 600), (13, 260, 279)])
def test_tiles_of_low_rank(shape, dtype):
    """Where what rounding loses is multiplied from step to step."""
    count, rows, cols = shape
    g = (torch.randn(count, rows, 8, device="cuda") @ torch.randn(count, 8, cols, device="cuda")).to(dtype)
    assert worst(dsm.orthogonalize(g), orth64(g)) < TOL_LOW_RANK[dtype]
