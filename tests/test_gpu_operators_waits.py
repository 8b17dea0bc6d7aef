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


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_without_its_products_is_nan(shape, dtype, monkeypatch):
    """Without a workspace of the caller's the results alone can tell.  Nothing beside them is written."""
    count, rows, cols = shape
    g, m = torch.randn(shape, device="cuda").to(dtype), torch.zeros(shape, device="cuda")
    wide = torch.full((count, rows + 2, cols + 5), 7.0, dtype=dtype, device="cuda")
    out, turned = wide[:, 1:-1, 3:-2], torch.zeros(count, cols, rows, dtype=dtype, device="cuda").mT
    monkeypatch.setenv("DSM_INJECT_OPERATOR_TIMEOUT", "1")
    dsm.orthogonalize(g, momentum=m, out=out)
    dsm.orthogonalize(g, out=turned)
    assert bool(out.isnan().all()) and bool(turned.isnan().all())
    assert int(wide.isnan().sum()) == out.numel() and bool((m == g.float()).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [0, 60, 200])
def test_linear_cross_entropy_without_its_products_is_nan(tokens, dtype, monkeypatch):
    h, w, y, a = problem(tokens, 700, 72, dtype, 0.2)
    _, right = dsm.linear_cross_entropy(h, w, y)
    wide_h = torch.full((tokens, 80), 7.0, dtype=dtype, device="cuda")
    wide_w = torch.full((702, 75), 7.0, dtype=dtype, device="cuda")
    out_h, out_w = wide_h[:, 5:77], wide_w[1:-1, 1:73]
    monkeypatch.setenv("DSM_INJECT_OPERATOR_TIMEOUT", "1")
    loss, lse = dsm.linear_cross_entropy(h, w, y)
    assert bool(loss.isnan().all()) and bool(lse.isnan().all())
    for need_h, need_w in ((True, True), (True, False), (False, True)):
        wide_h.fill_(7), wide_w.fill_(7)
        dsm.linear_cross_entropy_grad(h, w, y, right, a, out_h=out_h, out_weight=out_w, need_h=need_h, need_weight=need_w)
        assert int(wide_h.isnan().sum()) == int(out_h.isnan().sum()) == out_h.numel() * need_h
        assert int(wide_w.isnan().sum()) == int(out_w.isnan().sum()) == out_w.numel() * need_w


def test_a_loss_under_autograd_without_its_products_is_nan(monkeypatch):
    h, w, y, _ = problem(60, 700, 72, F32)
    h.requires_grad_(), w.requires_grad_()
    monkeypatch.setenv("DSM_INJECT_OPERATOR_TIMEOUT", "1")
    loss = dsm.linear_cross_entropy_loss(h, w, y)
    loss.backward()
    assert bool(loss.detach().isnan()) and bool(h.grad.isnan().all()) and bool(w.grad.isnan().all())
