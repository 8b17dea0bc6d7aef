"""linear_cross_entropy_loss under autograd: what it cannot do it refuses."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2411_17866_gb300 import dsm  # noqa: E402
from test_gpu_operators import TOL_GRAD, ce64, problem, rel  # noqa: E402

F32 = torch.float32


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.manual_seed(5)


@pytest.fixture
def leaf():
    h, w, y, _ = problem(50, 300, 64, F32, 0.2)
    h.requires_grad_(), w.requires_grad_()
    kept = max(1, int((y != -100).sum()))
    want = ce64(h.detach(), w.detach(), y, torch.full((1,), 1 / kept, device="cuda"))
    return h, w, y, want


def test_second_derivatives_are_refused(leaf):
    h, w, y, want = leaf
    loss = dsm.linear_cross_entropy_loss(h, w, y)
    dh, dw = torch.autograd.grad(loss, (h, w), create_graph=True)
    assert rel(dh.detach(), want[2]) < TOL_GRAD[F32] and rel(dw.detach(), want[3]) < TOL_GRAD[F32]
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (dh.square().sum() + dw.square().sum()).backward()


def test_a_penalty_on_the_gradient_is_refused_beside_a_loss(leaf):
    h, w, y, _ = leaf
    for inputs in ((h,), (w,), (h, w)):
        loss = dsm.linear_cross_entropy_loss(h, w, y)
        grads = torch.autograd.grad(loss, inputs, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(loss + sum(g.square().sum() for g in grads), h)
    # and by the incoming gradient alone
    s = torch.ones((), device="cuda", requires_grad=True)
    dh, = torch.autograd.grad(dsm.linear_cross_entropy_loss(h, w, y), h, grad_outputs=s, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(dh.sum(), s)


def test_a_recorded_backward_pass_gives_the_same_gradients(leaf):
    h, w, y, want = leaf
    out = torch.empty_like(w)
    dsm.linear_cross_entropy_loss(h, w, y, out_weight=out).backward(create_graph=True)
    assert rel(h.grad.detach(), want[2]) < TOL_GRAD[F32] and rel(w.grad.detach(), want[3]) < TOL_GRAD[F32]
    assert torch.equal(out, w.grad.detach())
    h.grad = w.grad = None   # (a recorded gradient holds on to its graph)


def test_out_weight_that_is_the_weights_own_gradient_is_refused(leaf):
    """Autograd would add the tensor to itself: twice the gradient."""
    h, w, y, want = leaf
    flat = torch.zeros(w.numel() + 64, device="cuda")
    buf = flat[64:].view_as(w)
    w.grad = buf
    for out in (buf, flat[64:].view_as(w), flat[32:32 + w.numel()].view_as(w)):
        with pytest.raises(ValueError, match="weight.grad"):
            dsm.linear_cross_entropy_loss(h, w, y, out_weight=out).backward()
    assert bool((flat == 0).all())                          # nothing was written
    # another part of the same storage, no gradient yet, and no out_weight at all are fine
    both = torch.zeros(2, *w.shape, device="cuda")
    w.grad = both[0]
    dsm.linear_cross_entropy_loss(h, w, y, out_weight=both[1]).backward()
    assert torch.equal(both[0], both[1]) and rel(both[0], want[3]) < TOL_GRAD[F32]
    w.grad = None
    dsm.linear_cross_entropy_loss(h, w, y, out_weight=buf).backward()
    assert torch.equal(w.grad, buf) and rel(buf, want[3]) < TOL_GRAD[F32]
    w.grad = buf.zero_()
    dsm.linear_cross_entropy_loss(h, w, y).backward()
    assert w.grad is buf and rel(buf, want[3]) < TOL_GRAD[F32]


def test_two_losses_of_one_backward_pass_do_not_share_an_out_weight(leaf):
    h, w, y, want = leaf
    buf = torch.empty_like(w)
    two = dsm.linear_cross_entropy_loss(h, w, y, out_weight=buf) + dsm.linear_cross_entropy_loss(2 * h, w, y, out_weight=buf)
    with pytest.raises(ValueError, match="two losses"):
        two.backward()
    # one after the other they may
    h.grad = w.grad = None
    first, second = (dsm.linear_cross_entropy_loss(h, w, y, out_weight=buf) for _ in range(2))
    for loss in (first, second):
        w.grad = None
        loss.backward(retain_graph=True)
        assert rel(buf, want[3]) < TOL_GRAD[F32] and torch.equal(buf, w.grad)
    w.grad = None
    first.backward()
    assert torch.equal(buf, w.grad)


def test_a_weight_that_is_no_leaf_and_is_used_twice(leaf):
    """An embedding used for the lookup as well: both gradients add up, and out_weight holds the head's."""
    h, w, y, want = leaf
    buf = torch.empty_like(w)
    (dsm.linear_cross_entropy_loss(h, w * 1.0, y, out_weight=buf) + (3 * w).sum()).backward()
    assert rel(w.grad, want[3] + 3) < TOL_GRAD[F32] and rel(buf, want[3]) < TOL_GRAD[F32]
    w.grad = None
    (dsm.linear_cross_entropy_loss(h, w, y, out_weight=buf) + (3 * w).sum()).backward()
    assert rel(w.grad, want[3] + 3) < TOL_GRAD[F32] and rel(buf, want[3]) < TOL_GRAD[F32]


@pytest.mark.parametrize("tokens", [1, 3, 50])
def test_grad_loss_of_any_stride(tokens):
    """An expanded value is what autograd hands to the summands of a sum."""
    h, w, y, a = problem(tokens, 300, 64, F32)
    _, lse = dsm.linear_cross_entropy(h, w, y)
    apart = torch.stack((a, 7 * a), 1)[:, 0]
    one = a[:1].clone()
    for given, plain in ((apart, a), (one.expand(tokens), one.repeat(tokens)), (one[0], one.repeat(tokens))):
        want = dsm.linear_cross_entropy_grad(h, w, y, lse, plain.contiguous())
        got = dsm.linear_cross_entropy_grad(h, w, y, lse, given)
        assert all(torch.equal(x, z) for x, z in zip(got, want))


def test_a_sum_of_losses_under_a_function_of_the_callers():
    """The operator as the user's own autograd function has it: backward() of a sum brings an expanded gradient."""
    h, w, y, _ = problem(50, 300, 64, F32, 0.2)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, w):
            loss, lse = dsm.linear_cross_entropy(h, w, y)
            ctx.save_for_backward(h, w, lse)
            return loss

        @staticmethod
        def backward(ctx, grad):
            h, w, lse = ctx.saved_tensors
            return dsm.linear_cross_entropy_grad(h, w, y, lse, grad)

    h.requires_grad_(), w.requires_grad_()
    Loss.apply(h, w).sum().backward()
    want = ce64(h.detach(), w.detach(), y, torch.ones(1, device="cuda"))
    assert rel(h.grad, want[2]) < TOL_GRAD[F32] and rel(w.grad, want[3]) < TOL_GRAD[F32]
