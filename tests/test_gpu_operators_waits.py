"""A wait on the GPU that runs out ends its kernel, is reported, and leaves the workspace and the device usable.

DSM_INJECT_OPERATOR_TIMEOUT=1 makes the kernels act as if a wait had run out; on their way out they then wait, in vain and
for their limit (1.5 to 3 s), for what such a run might have under way.
"""
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


# one CTA and a cluster of CTAs per matrix, and the general way with single CTAs and pairs
SHAPES = [(2, 60, 60), (1, 100, 700), (1, 300, 400), (24, 600, 1000)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_reports_a_wait_that_ran_out(shape, dtype, monkeypatch):
    g = torch.randn(shape, device="cuda").to(dtype)
    ws = dsm.orthogonalize_workspace(g)
    monkeypatch.setenv("DSM_INJECT_OPERATOR_TIMEOUT", "1")
    dsm.orthogonalize(g, workspace=ws)
    assert dsm.operator_status(ws) == 1
    monkeypatch.delenv("DSM_INJECT_OPERATOR_TIMEOUT")
    assert rel(dsm.orthogonalize(g, workspace=ws), orth64(g)) < TOL[dtype]
    assert dsm.operator_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [60, 200])
def test_linear_cross_entropy_reports_a_wait_that_ran_out(tokens, dtype, monkeypatch):
    h, w, y, a = problem(tokens, 700, 72, dtype, 0.2)
    ws = dsm.linear_cross_entropy_workspace(h, w)
    monkeypatch.setenv("DSM_INJECT_OPERATOR_TIMEOUT", "1")
    _, lse = dsm.linear_cross_entropy(h, w, y, workspace=ws)
    assert dsm.operator_status(ws) == 1
    dsm.linear_cross_entropy_grad(h, w, y, lse, a, workspace=ws)
    assert dsm.operator_status(ws) == 1
    monkeypatch.delenv("DSM_INJECT_OPERATOR_TIMEOUT")
    check(h, w, y, a)
