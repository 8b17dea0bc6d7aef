"""The operators on values that lie far from the ordinary: logits far below zero, rows and entries of very different sizes.

Losses are held to 1e-5 of the largest logit, gradients to the bounds of test_gpu_operators.check(), unless a test says
more.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2411_17866_gb300 import dsm  # noqa: E402
from test_gpu_operators import ce64, check, orth64, problem, rel  # noqa: E402

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


# ---- f32 gradients, row by row, with rows of very different sizes -----------------------------------------------------

def rows_within_bounds(h, w, y, a, **kw):
    """f32 gradients against 64 bits, every row of dh and of dW by a bound of its own, from the formats alone.

    A logit is known to 2^-20 of the sum of its products' sizes (operands of 22 bits, three terms, f32 sums), and so is its
    probability; G and h keep 22 bits, and 2^-39 of the largest of a token (for dh) or of all (for dW) as an absolute
    error; products and sums of f32 add 2^-21 of the sum of their sizes."""
    kept = y != -100
    ak = torch.where(kept, a.double().expand(len(y)), 0.0)
    h64, w64 = torch.where(kept[:, None], h, 0).double(), w.double()
    p = torch.softmax(h64 @ w64.T, 1)
    size = (h64.abs() @ w64.abs().T).amax(1).clamp_min(1.0)
    g = p.clone()
    g[torch.arange(len(y), device="cuda"), y.clamp_min(0)] -= 1
    g *= ak[:, None]
    dh, dw = g @ w64, g.T @ h64
    off = ak.abs()[:, None] * p * (2.0 ** -20 * size)[:, None] + 2.0 ** -21 * g.abs()
    wn, hn = w64.norm(dim=1), h64.norm(dim=1)
    bound_h = off @ wn + 2.0 ** -39 * ak.abs() * len(w) * w.shape[1] ** 0.5 * float(w64.abs().max())
    bound_w = off.T @ hn + 2.0 ** -39 * float(ak.abs().max()) * hn.sum() \
        + 2.0 ** -39 * h.shape[1] ** 0.5 * float(h64.abs().max()) * g.abs().sum(0)

    ws = dsm.linear_cross_entropy_workspace(h, w)
    loss, lse = dsm.linear_cross_entropy(h, w, y, workspace=ws)
    got_h, got_w = dsm.linear_cross_entropy_grad(h, w, y, lse, a, workspace=ws, **kw)
    assert dsm.operator_status(ws) == 0
    assert bool(((got_h.double() - dh).norm(dim=1) <= bound_h).all())
    assert bool(((got_w.double() - dw).norm(dim=1) <= bound_w).all())
    return dh, dw, bound_h, bound_w


def _sizes(rows, exponents):
    """A factor of 2^e for three rows of every e."""
    f = torch.ones(rows, 1, device="cuda")
    for i, e in enumerate(exponents):
        f[5 + 7 * i:5 + 7 * i + 3] = 2.0 ** e
    return f


@pytest.mark.parametrize("tokens", [17, 100, 300])
@pytest.mark.parametrize("what", ["plain", "zero w", "zero h", "zero both", "all w zero", "all h zero", "small w", "small h",
                                  "small both", "large w", "large h", "spread a", "zero a", "tiny all", "large all"])
def test_rows_of_different_sizes(what, tokens):
    h, w, y, a = problem(tokens, 1030, 96, F32, lean=8.0)
    y[3] = -100
    if what in ("zero w", "zero both"):
        w[[0, 400, 1029]] = 0
    if what in ("zero h", "zero both"):
        h[[1, 7, tokens - 1]] = 0
    if what == "all w zero":
        w.zero_()
    if what == "all h zero":
        h.zero_()
    down, up = (-10, -20, -30, -60, -100), (4, 8)
    if what in ("small w", "small both"):
        w *= _sizes(len(w), down)
    if what in ("small h", "small both"):
        h *= _sizes(tokens, down)[:tokens]
    if what == "large w":
        w *= _sizes(len(w), up)
    if what == "large h":
        h *= _sizes(tokens, up)
    if what == "spread a":
        a *= 2.0 ** -torch.randint(0, 12, (tokens,), device="cuda")
    if what == "zero a":
        a[::2] = 0
    if what == "tiny all":
        h, w = h * 2.0 ** 90, w * 2.0 ** -90
    if what == "large all":
        h, w, a = h * 2.0 ** -100, w * 2.0 ** 100, a * 2.0 ** 20
    dh, dw, bound_h, bound_w = rows_within_bounds(h, w, y, a)
    if what in ("plain", "zero w", "zero h", "zero both", "small w"):
        # the bounds say something: 1e-4 of a row, for nearly all rows
        kept = y != -100
        assert float((bound_h < 1e-4 * dh.norm(dim=1))[kept].double().mean()) > 0.9
        assert float((bound_w < 1e-4 * dw.norm(dim=1)).double().mean()) > 0.9


def test_zero_rows_of_a_larger_problem():
    """A padding row in W at an odd offset, a zero row among the kept ones, and pieces of the vocabulary."""
    h, w, y, a = problem(509, 10007, 451, F32, 0.1, lean=8.0)
    w[17] = 0
    h[11] = 0
    y[11] = 5
    flat = torch.empty(3 + w.numel(), device="cuda")
    flat[3:] = w.reshape(-1)
    rows_within_bounds(h, flat[3:].view_as(w), y, a)
    h, w, y, a = problem(9000, 16000, 24, F32, 0.1)
    w[[0, 15999]] = 0
    check(h, w, y, a)


def test_one_of_the_gradients_with_rows_of_different_sizes():
    h, w, y, a = problem(200, 1030, 96, F32)
    w[:4] = 0
    _, lse = dsm.linear_cross_entropy(h, w, y)
    dh, dw = dsm.linear_cross_entropy_grad(h, w, y, lse, a)
    assert torch.equal(dsm.linear_cross_entropy_grad(h, w, y, lse, a, need_weight=False)[0], dh)
    assert torch.equal(dsm.linear_cross_entropy_grad(h, w, y, lse, a, need_h=False)[1], dw)


# ---- rows of W that share a direction ---------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 3, 16, 100, 300])
@pytest.mark.parametrize("shift", [-56, -88, -96, -120, -400])
def test_gradients_where_all_rows_share_a_direction(shift, tokens, dtype):
    """The gradient of the logits adds up to zero over the vocabulary, so what W's rows have in common is not in dh."""
    check(*shifted(tokens, 1030, 96, dtype, shift))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 60, 200])
def test_gradients_where_rows_of_a_large_vocabulary_share_a_direction(tokens, dtype):
    check(*shifted(tokens, 50257, 64, dtype, -120))
    check(*shifted(tokens, 50257, 64, dtype, -240, slice(7, 40000)))


def test_gradients_where_all_rows_share_a_direction_by_pieces_and_parts():
    """Sums over a row of G that several pieces of the vocabulary and several parts of it add to, with ignored tokens, W at
    an odd offset, and a gradient of one token far smaller than the others'."""
    h, w, y, a = shifted(9000, 33001, 64, BF16, -120)
    y[::3] = -100
    check(h, w, y, a)
    h, w, y, a = shifted(70, 9001, 101, BF16, -120)
    y[5] = -100
    a[6], a[7] = 0, 1e-30
    flat = torch.empty(1 + w.numel(), dtype=BF16, device="cuda")
    flat[1:] = w.reshape(-1)
    check(h, flat[1:].view_as(w), y, a)


# ---- orthogonalize: sizes near the ends of the formats' range ---------------------------------------------------------

ORTH_TOL = {BF16: 5e-3, F32: 1e-5}


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1024, 1024), (90, 200), (600, 60)])
@pytest.mark.parametrize("size", [1e-24, 1e-16, 1e6, 1e9, 1e16, 1e17, 1e18, 1e19, 1e25, 1e37])
def test_orthogonalize_of_any_size(size, rows, cols, dtype):
    """Squares and their sum, and the norm itself, may lie beyond f32's range."""
    g = (torch.randn(rows, cols, device="cuda").double() * size).to(dtype)
    assert rel(dsm.orthogonalize(g, eps=1e-30), orth64(g, eps=1e-30)) < ORTH_TOL[dtype]
    # no steps: one rounding of the result, and the norm's (sums of 10^6 squares in a few levels: 1e-6)
    assert rel(dsm.orthogonalize(g, 0, eps=1e-30), orth64(g, 0, eps=1e-30)) < (2.0 ** -8 if dtype == BF16 else 2e-6)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(300, 400), (100, 700)])
def test_orthogonalize_of_mixed_sizes(rows, cols, dtype):
    """Entries on both sides of where squares are summed apart, and some far above the others; with a momentum."""
    g = torch.randn(2, rows, cols, device="cuda")
    g[0, ::2] *= 2.0 ** 22
    g[1, :, ::3] *= 2.0 ** 23
    g[0, 0, :7] *= 2.0 ** 10
    g = g.to(dtype)
    m = torch.randn(2, rows, cols, device="cuda") * 2.0 ** 20
    want_m = float(torch.tensor(0.95)) * m.double() + g.double()
    want = orth64(g.double() + float(torch.tensor(0.95)) * want_m)
    assert rel(dsm.orthogonalize(g, momentum=m), want) < ORTH_TOL[dtype]
    assert rel(m, want_m) < 2.0 ** -22


def test_orthogonalize_zero_with_a_tiny_eps():
    for shape in ((200, 300), (60, 60)):
        g = torch.zeros(shape, device="cuda")
        for eps in (1e-7, 1e-30, 1e-38, 1e-44):
            assert bool((dsm.orthogonalize(g, eps=eps) == 0).all()) and bool((dsm.orthogonalize(g, 0, eps=eps) == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("shape", [(3, 130, 200), (3, 40, 90)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_orthogonalize_makes_a_matrix_that_is_not_finite_nan(bad, shape, steps, dtype):
    g = torch.randn(shape, device="cuda").to(dtype)
    g[1, 5, 7] = bad
    got = dsm.orthogonalize(g, steps)
    assert bool(got[1].isnan().all())
    for i in (0, 2):
        assert rel(got[i], orth64(g[i], steps)) < ORTH_TOL[dtype]


# ---- what the accumulators cut off ------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [60, 128, 200])
@pytest.mark.parametrize("vocab", [700, 50257])
@pytest.mark.parametrize("width", [512, 768, 1024, 1600, 2048])
def test_long_sums_of_one_sign(width, vocab, tokens):
    """Sums leave the accumulators every 512 k.  Until then each of 32 additions cuts off half of the last bit on average
    (2^-24 of the sum so far, which is half of the whole on average): the mean error of logits that are sums of one sign is
    below 16 * 2^-24, and it does not grow with the width."""
    h = torch.rand(tokens, width, device="cuda").to(BF16)
    w = (torch.rand(vocab, width, device="cuda") * (160 / width)).to(BF16)
    y = torch.randint(0, vocab, (tokens,), device="cuda")
    _, lse = dsm.linear_cross_entropy(h, w, y)
    want = torch.logsumexp(h.double() @ w.double().T, 1)
    assert abs(float(((lse.double() - want) / want).mean())) < 16 * 2.0 ** -24


# ---- f32 gradients of tokens that count for very different amounts ----------------------------------------------------

@pytest.mark.parametrize("tokens", [17, 100, 300])
@pytest.mark.parametrize("spread", [0, 15, 25, 35, 60])
def test_grad_loss_of_very_different_sizes(spread, tokens):
    """Tokens whose loss counts for little, beside sure ones that count for much and touch few rows of dW: the other rows are
    the small tokens' alone.  Bounds as in rows_within_bounds(), but absolutely only 2^-39 of each token's own grad_loss_t h_t
    (and not more than its G there), and 2^-39 of the largest value of grad_loss_t h_t times G."""
    h, w, y, a = problem(tokens, 1030, 96, F32, lean=4.0)
    big = torch.arange(tokens, device="cuda") % 4 == 0
    y[big] %= 10
    w[:10] *= 20
    h[big] = (h + 3 * w[y])[big]
    a[~big] *= 2.0 ** -spread
    h64, w64, a64 = h.double(), w.double(), a.double()
    z = h64 @ w64.T
    p = torch.softmax(z, 1)
    size = torch.maximum((h64.abs() @ w64.abs().T).amax(1), torch.logsumexp(z, 1).abs()).clamp_min(1.0)
    q = p.clone()
    q[torch.arange(tokens, device="cuda"), y] -= 1
    dh, dw = a64[:, None] * (q @ w64), q.T @ (a64[:, None] * h64)
    off = p * (2.0 ** -20 * size)[:, None] + 2.0 ** -21 * q.abs()
    ah = a64 * h64.norm(dim=1)
    bound_h = a64 * (off @ w64.norm(dim=1) + 2.0 ** -39 * len(w) * 96 ** 0.5 * float(w64.abs().max()))
    bound_w = (off + q.abs().clamp_max(2.0 ** -39)).T @ ah + 2.0 ** -39 * 96 ** 0.5 * float((a64[:, None] * h64).abs().max()) * q.abs().sum(0)
    _, lse = dsm.linear_cross_entropy(h, w, y)
    got_h, got_w = dsm.linear_cross_entropy_grad(h, w, y, lse, a)
    assert bool(((got_h.double() - dh).norm(dim=1) <= bound_h).all())
    assert bool(((got_w.double() - dw).norm(dim=1) <= bound_w).all())


# ---- sure tokens ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", [(3, 20, 1600), (8, 20, 1600), (8, 20, 520), (17, 20, 1100), (60, 90, 1900), (140, 20, 1600),
                                                (300, 1030, 4096)])
def test_tokens_that_are_sure(tokens, vocab, width, dtype):
    """Logits that are nearly all of lse: what is left of p - 1 shows whether the gradient forms them as the loss did."""
    for _ in range(30 if tokens < 100 else 5):
        check(*problem(tokens, vocab, width, dtype, 0.5 if tokens > 3 else 0.0, lean=20.0 if width < 4000 else 6.0))


@pytest.mark.parametrize("tokens", [60, 200])
@pytest.mark.parametrize("vocab", [700, 10007])
@pytest.mark.parametrize("width", [256, 768, 1024, 1600])
def test_long_f32_sums_of_one_sign(width, vocab, tokens):
    """f32 operands: sums leave the accumulators every 64 k, within which the four large additions of 16 k cut off 2^-24 of the sum
    so far on average, 2.5 * 2^-24 of a whole (1/4 + 2/4 + 3/4 + 1); those before, with lo, nearly nothing."""
    h = torch.rand(tokens, width, device="cuda")
    w = torch.rand(vocab, width, device="cuda") * (160 / width)
    y = torch.randint(0, vocab, (tokens,), device="cuda")
    _, lse = dsm.linear_cross_entropy(h, w, y)
    want = torch.logsumexp(h.double() @ w.double().T, 1)
    assert abs(float(((lse.double() - want) / want).mean())) < 4 * 2.0 ** -24
