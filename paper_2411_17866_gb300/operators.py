"""The operators next to the rounds as torch functions: argument marshalling for include/dsm.h, no arithmetic.

``linear_cross_entropy`` and its gradient are the loss of a language-model head (h W^T against targets) without the
logits being kept; ``orthogonalize`` turns a weight matrix's gradient, with its momentum, into an orthogonalised update
direction.  Everything runs in the library's CUDA kernels on torch's current stream (or ``stream``); torch supplies the
memory of outputs and workspaces, unless they are given.  All names are reached through the ``dsm`` module as well.

A tensor that is used on another stream than the one it was allocated on is the caller's to keep alive (torch's
``record_stream``), except for what these functions allocate themselves.
"""
from __future__ import annotations

import ctypes
from ctypes import byref

from . import dsm as _d

#: One Newton-Schulz step's (a, b, c): the quintic that takes singular values in (0, 1] to about 1 in five steps.
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


torch = None   # the module, once a function has been called (importing this module does not import it)
_DTYPES = {}


def _import_torch():
    global torch
    if torch is None:
        import torch as module
        _DTYPES.update({module.bfloat16: _d.BF16, module.float32: _d.F32})
        torch = module


def _dtype_of(t, name):
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}") from None


def _on_gpu(**tensors):
    """Checks that all tensors lie on one CUDA device, and returns its index."""
    if torch is None:
        _import_torch()
    index = None
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        i = t.get_device()
        if index is None:
            index = i
        elif i != index:
            raise ValueError(f"{name} is on device {i}, other arguments are on device {index}")
    return index


_functions = {}


def _call(index, func, *args, stream):
    """Calls the library with device `index` as the current one and ``stream``, torch's current one if None."""
    call = _functions.get(func)
    if call is None:
        call = _functions[func] = getattr(_d.load_library(), func)
    if torch.cuda.current_device() == index:
        rc = call(*args, _d._stream(stream))
    else:
        with torch.cuda.device(index):   # 2 us: only where it is not current
            rc = call(*args, _d._stream(stream))
    if rc != _d.DSM_OK:
        _d._check(rc, func)


def _new(shape, dtype, index, stream):
    """A new tensor that stays allocated until ``stream`` is done with it."""
    t = torch.empty(shape, dtype=dtype, device=index)
    if stream is not None:
        s = stream if not isinstance(stream, int) else torch.cuda.ExternalStream(stream, device=index)
        s.wait_stream(torch.cuda.current_stream(index))   # the memory's earlier use
        t.record_stream(s)
    return t


def _given(workspace, index):
    if not workspace.is_cuda or workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the other arguments")
    return workspace


def operator_status(workspace, stream=None) -> int:
    """0, or 1 if a wait of the last operator call on this workspace ran out on the GPU (what it has not computed is then NaN,
    as it is where no workspace was given).  Synchronises the stream."""
    out = ctypes.c_uint32()
    rc = _d.load_library().dsm_operator_status(workspace.data_ptr(), _d._stream(stream), byref(out))
    _d._check(rc, "dsm_operator_status")
    return out.value


# ---- orthogonalised updates ---------------------------------------------------------------------------------------

def _strides(t):
    s = t.stride()
    return (ctypes.c_int64 * 3)(*(s if t.dim() == 3 else (0, *s)))


def _orth_args(g, out, momentum, steps, coefficients, mu, nesterov, eps, scale):
    if g.dim() not in (2, 3):
        raise ValueError("g must have two dimensions (a matrix) or three (a stack of matrices)")
    dtype = _dtype_of(g, "g")
    if out is not None and (out.shape != g.shape or out.dtype != g.dtype):
        raise ValueError("out must have the shape and type of g")
    if momentum is not None and (momentum.shape != g.shape or momentum.dtype != torch.float32):
        raise ValueError("momentum must be float32 with the shape of g")
    a = _d.dsm_orthogonalize_args()
    a.dtype = dtype
    a.count = 1 if g.dim() == 2 else g.shape[0]
    a.rows, a.cols = g.shape[-2], g.shape[-1]
    a.steps = steps
    if len(coefficients) == 3 and not hasattr(coefficients[0], "__len__"):
        flat = tuple(coefficients) * steps
    else:
        if len(coefficients) != steps:
            raise ValueError("coefficients must be one (a, b, c), or one for every step")
        flat = tuple(v for step in coefficients for v in step)
    a._keep = (ctypes.c_float * len(flat))(*flat)
    a.coefficients = ctypes.cast(a._keep, ctypes.POINTER(ctypes.c_float))
    a.g, a.g_stride = g.data_ptr(), _strides(g)
    if out is not None:
        a.out, a.out_stride = out.data_ptr(), _strides(out)
    if momentum is not None:
        a.momentum, a.momentum_stride = momentum.data_ptr(), _strides(momentum)
    a.mu, a.nesterov, a.eps, a.scale = mu, int(bool(nesterov)), eps, scale
    return a


def orthogonalize_workspace(g):
    """A workspace (uint8 tensor) for ``orthogonalize`` on a tensor like ``g``."""
    index = _on_gpu(g=g)
    a = _orth_args(g, None, None, 1, COEFFICIENTS, 0.0, False, 1e-7, 1.0)
    return torch.empty(_orth_bytes(a), dtype=torch.uint8, device=index)


def _orth_bytes(a):
    n = _d.load_library().dsm_orthogonalize_workspace(byref(a))
    if n == 0:
        raise _d.DsmError(_d.DSM_EINVAL, "dsm_orthogonalize_workspace", _d.last_error())
    return n


def orthogonalize(g, steps=5, *, coefficients=COEFFICIENTS, momentum=None, mu=0.95, nesterov=True, eps=1e-7, scale=1.0,
                  out=None, workspace=None, stream=None):
    """Newton-Schulz orthogonalisation of a matrix, or of each matrix of a stack, of any strides.

    With ``momentum`` (float32, updated in place): momentum <- mu momentum + g, and g + mu momentum (``nesterov``) or
    momentum takes the place of g.  Then X = u / max(|u|, eps), ``steps`` times X <- a X + (b A + c A A) X with
    A = X X^T, and ``scale`` X is returned in ``out`` (a new tensor of g's type if not given; it may be g).
    ``coefficients``: one (a, b, c), or one for every step.
    """
    index = _on_gpu(g=g, out=out, momentum=momentum)
    if out is None:
        out = _new(g.shape, g.dtype, index, stream)
    a = _orth_args(g, out, momentum, steps, coefficients, mu, nesterov, eps, scale)
    ws = _new(_orth_bytes(a), torch.uint8, index, stream) if workspace is None else _given(workspace, index)
    _call(index, "dsm_orthogonalize", byref(a), ws.data_ptr(), ws.nbytes, stream=stream)
    return out


# ---- linear cross entropy -----------------------------------------------------------------------------------------

def _rows(t, name, shape=None):
    """The stride of a matrix's rows, whose elements must lie next to each other."""
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be a matrix" + (f" of {tuple(shape)}" if shape is not None else ""))
    rows, columns = t.stride()
    if columns != 1 and t.shape[1] > 1:
        raise ValueError(f"the elements of a row of {name} must lie next to each other (stride 1)")
    return rows


def _ce_args(h, weight, targets, ignore_index):
    dtype = _dtype_of(h, "h")
    if weight.dtype != h.dtype:
        raise ValueError("h and weight must have the same type")
    h_stride, w_stride = _rows(h, "h"), _rows(weight, "weight")
    tokens, width = h.shape
    vocab, weight_width = weight.shape
    if weight_width != width:
        raise ValueError(f"weight must have the {width} columns of h, not {weight_width}")
    at, size = None, 8
    if targets is not None:
        if targets.shape != (tokens,) or not targets.is_contiguous():
            raise ValueError("targets must be a contiguous vector with one entry per row of h")
        if targets.dtype not in (torch.int64, torch.int32):
            raise ValueError(f"targets must be int64 or int32, not {targets.dtype}")
        at, size = targets.data_ptr(), targets.element_size()
    return _d.dsm_linear_ce(h.data_ptr(), weight.data_ptr(), at, h_stride, w_stride, ignore_index, tokens, vocab, width,
                            dtype, size, 0)


def _ce_bytes(a, grad):
    n = _d.load_library().dsm_linear_cross_entropy_workspace(byref(a), int(bool(grad)))
    if n == 0:
        raise _d.DsmError(_d.DSM_EINVAL, "dsm_linear_cross_entropy_workspace", _d.last_error())
    return n


def linear_cross_entropy_workspace(h, weight, grad=True):
    """A workspace (uint8 tensor) for ``linear_cross_entropy`` and, with ``grad``, ``linear_cross_entropy_grad``."""
    index = _on_gpu(h=h, weight=weight)
    a = _ce_args(h, weight, None, -100)
    nbytes = max(_ce_bytes(a, False), _ce_bytes(a, True) if grad else 0)
    return torch.empty(nbytes, dtype=torch.uint8, device=index)


def _vector(t, tokens, name):
    if t.shape != (tokens,) or t.dtype != torch.float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 vector with one entry per row of h")
    return t


def linear_cross_entropy(h, weight, targets, *, ignore_index=-100, workspace=None, stream=None):
    """Per-token cross entropy of the logits h weight^T against ``targets``: (loss, lse), float32, with lse the
    log-sum-exp of every token's logits.  Both are 0 where the target is ``ignore_index``, and NaN where it is neither
    that nor a row of ``weight``."""
    index = _on_gpu(h=h, weight=weight, targets=targets)
    a = _ce_args(h, weight, targets, ignore_index)
    loss, lse = _new(a.tokens, torch.float32, index, stream), _new(a.tokens, torch.float32, index, stream)
    ws = _new(_ce_bytes(a, False), torch.uint8, index, stream) if workspace is None else _given(workspace, index)
    _call(index, "dsm_linear_cross_entropy", byref(a), loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.nbytes,
          stream=stream)
    return loss, lse


def linear_cross_entropy_grad(h, weight, targets, lse, grad_loss, *, ignore_index=-100, out_h=None, out_weight=None,
                              need_h=True, need_weight=True, workspace=None, stream=None):
    """The gradients (of h, of weight) of sum(grad_loss * loss), from the ``lse`` of ``linear_cross_entropy``.

    ``grad_loss``: one float32 value per token (a vector of any stride, an expanded one too), or a tensor with one for all.  ``out_h`` and ``out_weight`` (rows of
    any stride: a worker's gradient buffer, say) are written whole; new tensors if not given.  A gradient that is not
    needed (``need_h``, ``need_weight``) is not computed, and None is returned for it."""
    index = _on_gpu(h=h, weight=weight, targets=targets, lse=lse, grad_loss=grad_loss, out_h=out_h,
                    out_weight=out_weight)
    a = _ce_args(h, weight, targets, ignore_index)
    _vector(lse, a.tokens, "lse")
    if grad_loss.dtype != torch.float32 or (grad_loss.numel() != 1 and grad_loss.shape != (a.tokens,)):
        raise ValueError("grad_loss must be a float32 vector with one entry per row of h, or one value")
    grad_stride = 0 if grad_loss.numel() == 1 else grad_loss.stride(0)

    def output(needed, given, like, name):
        if not needed:
            return None, None, 0
        if given is None:
            given = _new(like.shape, like.dtype, index, stream)
        elif given.dtype != like.dtype:
            raise ValueError(f"{name} must have the type of what it is the gradient of")
        return given, given.data_ptr(), _rows(given, name, like.shape)

    out_h, dh, dh_stride = output(need_h, out_h, h, "out_h")
    out_weight, dw, dw_stride = output(need_weight, out_weight, weight, "out_weight")
    if need_weight or (need_h and a.tokens):
        ws = _new(_ce_bytes(a, True), torch.uint8, index, stream) if workspace is None else _given(workspace, index)
        _call(index, "dsm_linear_cross_entropy_grad", byref(a), lse.data_ptr(), grad_loss.data_ptr(), grad_stride, dh,
              dh_stride, dw, dw_stride, ws.data_ptr(), ws.nbytes, stream=stream)
    return out_h, out_weight


def linear_cross_entropy_loss(h, weight, targets, *, ignore_index=-100, out_weight=None):
    """The mean loss over the tokens that are not ignored (0 if all are), differentiable in h and weight, once: second
    derivatives raise an error.

    ``out_weight``: where the gradient of ``weight`` is written in the backward pass (its slice of a worker's gradient
    buffer, say); autograd returns that tensor as the gradient.  ``weight.grad`` must not lie in the same memory, nor two
    losses of one backward pass write to it: autograd would add the tensor to itself (ValueError).  A gradient that
    autograd is to collect in ``weight.grad``, whatever its memory, needs no ``out_weight``."""
    return _function().apply(h, weight, targets, ignore_index, out_weight)


def _span(t):
    """The addresses from a tensor's first element to behind its last."""
    start = t.data_ptr()
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
    return (start, start + (last + 1) * t.element_size()) if t.numel() else (start, start)


def _overlap(a, b):
    return a[0] < b[1] and b[0] < a[1]


_pass, _pass_spans = None, []   # the last backward pass, and where it has written an out_weight


def _check_out_weight(weight, out):
    """Refuses an out_weight that autograd would add to itself."""
    global _pass, _pass_spans
    span = _span(out)
    if weight.is_leaf and weight.grad is not None and _overlap(_span(weight.grad), span):
        raise ValueError("weight.grad shares memory with out_weight, and autograd would add the gradient to itself: set "
                         "weight.grad to None before the backward pass, or leave out_weight out")
    current = torch._C._current_graph_task_id()
    if current != _pass:
        _pass, _pass_spans = current, []
    if any(_overlap(span, other) for other in _pass_spans):
        raise ValueError("two losses of one backward pass write to the same out_weight")
    _pass_spans.append(span)


_loss_function = None


def _function():
    """The autograd function behind linear_cross_entropy_loss (defined on first use: torch is imported lazily)."""
    global _loss_function
    if _loss_function is None:
        _import_torch()

        class Once(torch.autograd.Function):
            """Gradients as they are, for a backward pass that is itself recorded: differentiating them is an error, not
            nothing.  (torch's once_differentiable records them only where the incoming gradient requires one.)"""

            @staticmethod
            def forward(ctx, h, weight, grad, dh, dw):
                return tuple(None if g is None else g.detach() for g in (dh, dw))

            @staticmethod
            def backward(ctx, *grads):
                raise RuntimeError("linear_cross_entropy_loss is once_differentiable: it has no second derivatives")

        class LinearCrossEntropy(torch.autograd.Function):
            @staticmethod
            def forward(ctx, h, weight, targets, ignore_index, out_weight):
                loss, lse = linear_cross_entropy(h, weight, targets, ignore_index=ignore_index)
                kept = (targets != ignore_index).sum().clamp_min(1).to(torch.float32)
                ctx.save_for_backward(h, weight, targets, lse, kept)
                ctx.ignore_index, ctx.out_weight = ignore_index, out_weight
                return loss.sum() / kept

            @staticmethod
            def backward(ctx, grad):
                h, weight, targets, lse, kept = ctx.saved_tensors
                each = (grad.to(torch.float32) / kept).reshape(1)
                need_h, need_weight = ctx.needs_input_grad[:2]
                if need_weight and ctx.out_weight is not None:
                    _check_out_weight(weight, ctx.out_weight)
                dh, dw = linear_cross_entropy_grad(h, weight, targets, lse, each, ignore_index=ctx.ignore_index,
                                                   out_weight=ctx.out_weight, need_h=need_h, need_weight=need_weight)
                if torch.is_grad_enabled():
                    dh, dw = Once.apply(h, weight, grad, dh, dw)
                return dh, dw, None, None, None

        _loss_function = LinearCrossEntropy
    return _loss_function
