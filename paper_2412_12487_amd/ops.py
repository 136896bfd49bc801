"""Operators of a training step (include/echo_ops.h): embedding, layer norm and cross entropy, each
with its gradient, as HIP kernels of libecho.so.

The composer plans a job from its operators' durations; these are the operators of a pipeline
stage outside its matrix products, on the GPU at hand (`workloads.measured` times them for a graph).

    y = layer_norm(x, weight, bias)["y"]
    h = embedding(ids, table, scale)
    r = cross_entropy(logits, targets, grad_loss=g)          # loss, lse and the logits' gradient

Activations are float32, float16 or bfloat16 matrices whose rows are contiguous (leading dimensions in
one stride; nothing is copied into order behind the caller's back: another layout raises EchoError).
Sums and statistics are in 32 bits and each result is rounded once.  Work is enqueued on the
current stream of the tensors' GPU; outputs and workspaces not passed in come from torch's allocator on
that stream.  Every call can be captured in a HIP graph.  Results do not vary from run to run.

Nothing is recorded for automatic differentiation: gradients are calls of their own, and tensors that require grad
are taken under torch.no_grad() or detached (where a graph is recorded they raise EchoError).  Tensors that a call
writes over count as modified in place.
"""
from __future__ import annotations

import ctypes

import torch

from .echo import ECHO_ERR_ARG, EchoError, _check, lib

EXPORTS = ("echo_layer_norm", "echo_layer_norm_grad", "echo_layer_norm_grad_workspace", "echo_embedding",
           "echo_embedding_grad", "echo_embedding_grad_workspace", "echo_cross_entropy", "echo_cross_entropy_grad")

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_INDEX = {torch.int32: 0, torch.int64: 1}

_fns = None


def _ops():
    """The library with the operators' signatures set: each once and to what it stays, since two threads may get here
    together, and one go on to calls while the other sets them again."""
    global _fns
    if _fns is None:
        L = lib()
        P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        for name, restype, argtypes in (
                ("layer_norm", i32, [P, i64, P, i64, P, P, i32, i32, i64, i64, f32, P, P, P, P, i32, P]),
                ("layer_norm_grad", i32, [P, i64, P, i64, P, P, P, P, i64, i32, i32, i64, i64, P, P, P, i32, i32, P, i64, i32,
                                          P]),
                ("layer_norm_grad_workspace", i64, [i64, i64]),
                ("embedding", i32, [P, i32, P, i64, i32, i64, i64, i64, i64, f32, P, i32, P]),
                ("embedding_grad", i32, [P, i32, P, i64, i32, i64, i64, i64, i64, f32, P, i32, i32, P, i64, i32, P]),
                ("embedding_grad_workspace", i64, [i64, i64, i64]),
                ("cross_entropy", i32, [P, i64, i32, P, i32, i64, i64, i64, i64, P, P, P, P, P, i64, i32, P]),
                ("cross_entropy_grad", i32, [P, i64, i32, P, i32, i64, i64, i64, i64, P, P, P, i64, i32, P])):
            f = getattr(L, "echo_" + name)
            f.restype, f.argtypes = restype, argtypes
        _fns = L
    return _fns


def _bad(msg):
    return EchoError(ECHO_ERR_ARG, msg)


def _int64(n, name):
    """n as the library takes it; ctypes would cut a larger one."""
    n = int(n)
    if not -(1 << 63) <= n < 1 << 63:
        raise _bad(f"{name} = {n} does not fit 64 bits")
    return n


def _gpu(t, name):
    """Device index of the call's first tensor."""
    if not isinstance(t, torch.Tensor):
        raise _bad(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise _bad(f"{name} is on {t.device}: the operators run on the GPU")
    return t.device


_GRAPH = "%s requires grad, and the operators record no graph: call them under torch.no_grad() or with detached tensors"


def _matrix(t, name, dev, types):
    """(rows, cols, row stride) of a tensor read as rows of its last dimension."""
    if not isinstance(t, torch.Tensor):
        raise _bad(f"{name} must be a torch tensor")
    if t.device != dev:
        raise _bad(f"{name} is on {t.device}, the call on {dev}")
    if t.dtype not in types:
        raise _bad(f"{name} must be {' or '.join(str(x) for x in types)} (got {t.dtype})")
    if t.requires_grad and torch.is_grad_enabled():
        raise _bad(_GRAPH % name)
    if t.dim() < 1:
        raise _bad(f"{name} must have at least one dimension")
    cols = t.shape[-1]
    if cols < 1:
        raise _bad(f"{name} has rows of no elements")
    rows = t.numel() // cols
    if t.is_contiguous():
        return rows, cols, cols
    if rows <= 1:
        if rows and cols > 1 and t.stride(-1) != 1:
            raise _bad(f"{name}: the elements of a row must be contiguous (stride {t.stride(-1)})")
        return rows, cols, cols
    if cols > 1 and t.stride(-1) != 1:
        raise _bad(f"{name}: the elements of a row must be contiguous (stride {t.stride(-1)})")
    stride = n = None
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride, n = step, size
        elif step != stride * n:
            raise _bad(f"{name}: the leading dimensions {tuple(t.shape[:-1])} are not one run of rows "
                       f"(strides {t.stride()[:-1]})")
        else:
            n *= size
    return rows, cols, stride


def _vector(t, name, dev, n, types):
    if not isinstance(t, torch.Tensor):
        raise _bad(f"{name} must be a torch tensor")
    if t.device != dev:
        raise _bad(f"{name} is on {t.device}, the call on {dev}")
    if t.dtype not in types:
        raise _bad(f"{name} must be {' or '.join(str(x) for x in types)} (got {t.dtype})")
    if t.requires_grad and torch.is_grad_enabled():
        raise _bad(_GRAPH % name)
    if t.numel() != n:
        raise _bad(f"{name} has {t.numel()} elements, needs {n}")
    if not t.is_contiguous():
        raise _bad(f"{name} must be contiguous")
    return t.data_ptr()


def _like(t):
    """A new dense tensor like t."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _row(t, cols, dtype):
    """A new dense row of `cols` elements.  empty_like, where t is one, takes half of new_empty's time (1.1 of
    2.1 us on the host), which is much of a small call."""
    return torch.empty_like(t) if t.dtype == dtype and t.dim() == 1 else t.new_empty((cols,), dtype=dtype)


def _dense(t, name, dev, shape, dtype):
    """An output that the caller supplies, checked."""
    if not isinstance(t, torch.Tensor):
        raise _bad(f"{name} must be a torch tensor")
    if t.device != dev:
        raise _bad(f"{name} is on {t.device}, the call on {dev}")
    if t.dtype != dtype:
        raise _bad(f"{name} must be {dtype} (got {t.dtype})")
    if t.requires_grad and torch.is_grad_enabled():
        raise _bad(_GRAPH % name)
    if t.shape != torch.Size(shape):
        raise _bad(f"{name} has shape {tuple(t.shape)}, needs {tuple(shape)}")
    if not t.is_contiguous():
        raise _bad(f"{name} must be contiguous")
    return t


def _space(workspace, need, like):
    """Scratch of at least `need` bytes on like's GPU: the caller's, or a new one."""
    if workspace is None:
        return like.new_empty((need,), dtype=torch.uint8) if need else None
    if not isinstance(workspace, torch.Tensor) or workspace.device != like.device or not workspace.is_contiguous():
        raise _bad(f"workspace must be a contiguous tensor on {like.device}")
    return workspace


def _space_args(space):
    return (None, 0) if space is None else (space.data_ptr(), space.numel() * space.element_size())


# Handle of the current stream of GPU `index`: torch.cuda.current_stream(...).cuda_stream without the
# Stream object around it (1.7 us, a tenth of a small call)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _only(out, names):
    if not out:
        return {}
    out = dict(out)
    for k in out:
        if k not in names:
            raise _bad(f"out has no entry {k!r} here (entries: {', '.join(names)})")
    return out


# Counts tensors as modified in place, so that a backward pass that saved one of them notices.
_written = torch.autograd.graph.increment_version


def layer_norm(x, weight, bias=None, eps=1e-5, *, residual=None, out=None):
    """Layer norm over the last dimension, of x or of x + residual.

    Returns a dict: 'y' and, with a residual, 'sum' (x + residual, what is normalised), both like x;
    'mean' and 'rstd' float32 of x's leading shape, for layer_norm_grad.  `out` may supply tensors of
    those names ('sum' may be x or residual itself).  weight and bias: x's type or float32."""
    dev = _gpu(x, "x")
    rows, cols, xs = _matrix(x, "x", dev, _TYPES)
    w = _vector(weight, "weight", dev, cols, (x.dtype, torch.float32))
    b = None if bias is None else _vector(bias, "bias", dev, cols, (weight.dtype,))
    res = _only(out, ("y", "sum", "mean", "rstd") if residual is not None else ("y", "mean", "rstd"))
    r, rs = None, 0
    if residual is not None:
        if not isinstance(residual, torch.Tensor) or residual.shape != x.shape:
            raise _bad("residual must be a tensor of x's shape")
        _, _, rs = _matrix(residual, "residual", dev, (x.dtype,))
        r = residual.data_ptr()
        res["sum"] = _dense(res["sum"], "sum", dev, x.shape, x.dtype) if "sum" in res else _like(x)
    res["y"] = _dense(res["y"], "y", dev, x.shape, x.dtype) if "y" in res else _like(x)
    lead = x.shape[:-1]
    res["mean"] = (_dense(res["mean"], "mean", dev, lead, torch.float32) if "mean" in res
                   else x.new_empty(lead, dtype=torch.float32))
    res["rstd"] = (_dense(res["rstd"], "rstd", dev, lead, torch.float32) if "rstd" in res
                   else torch.empty_like(res["mean"]))
    _check(_ops().echo_layer_norm(
        x.data_ptr(), xs, r, rs, w, b, _TYPES[x.dtype], _TYPES[weight.dtype], rows, cols, float(eps),
        res["y"].data_ptr(), None if r is None else res["sum"].data_ptr(), res["mean"].data_ptr(),
        res["rstd"].data_ptr(), dev.index, _stream(dev.index)))
    if out:
        _written([res[k] for k in out])
    return res


def layer_norm_grad(dy, x, weight, mean, rstd, *, grad_residual=None, bias=True, dtype=None, out=None,
                    accumulate=False, workspace=None):
    """Gradients of layer_norm from that of y; x is what was normalised ('sum' where a residual was added).

    Returns a dict: 'dx' like x (plus grad_residual, the gradient that reaches x past the norm), 'dweight' and, unless
    bias=False, 'dbias', of weight's type or of `dtype` (float32).  `out` may supply tensors of those names
    ('dx' may be dy or grad_residual itself); with accumulate=True it has to supply 'dweight' (and 'dbias'),
    which are added to."""
    dev = _gpu(dy, "dy")
    rows, cols, ds = _matrix(dy, "dy", dev, _TYPES)
    if not isinstance(x, torch.Tensor) or x.shape != dy.shape:
        raise _bad("x must be a tensor of dy's shape")
    _, _, xs = _matrix(x, "x", dev, (dy.dtype,))
    w = _vector(weight, "weight", dev, cols, (dy.dtype, torch.float32))
    m = _vector(mean, "mean", dev, rows, (torch.float32,))
    k = _vector(rstd, "rstd", dev, rows, (torch.float32,))
    r, rs = None, 0
    if grad_residual is not None:
        if not isinstance(grad_residual, torch.Tensor) or grad_residual.shape != dy.shape:
            raise _bad("grad_residual must be a tensor of dy's shape")
        _, _, rs = _matrix(grad_residual, "grad_residual", dev, (dy.dtype,))
        r = grad_residual.data_ptr()
    names = ("dweight", "dbias") if bias else ("dweight",)
    res = _only(out, ("dx",) + names)
    if accumulate and any(n not in res for n in names):
        raise _bad(f"accumulate adds to out's {' and '.join(names)}")
    if dtype is None:
        dtype = res["dweight"].dtype if isinstance(res.get("dweight"), torch.Tensor) else weight.dtype
    if dtype not in (weight.dtype, torch.float32):
        raise _bad(f"dtype must be {weight.dtype} or torch.float32 (got {dtype})")
    res["dx"] = _dense(res["dx"], "dx", dev, dy.shape, dy.dtype) if "dx" in res else _like(dy)
    for n in names:
        res[n] = _dense(res[n], n, dev, (cols,), dtype) if n in res else _row(weight, cols, dtype)
    L = _ops()
    space = _space(workspace, L.echo_layer_norm_grad_workspace(rows, cols), dy)
    _check(L.echo_layer_norm_grad(
        dy.data_ptr(), ds, x.data_ptr(), xs, w, m, k, r, rs, _TYPES[dy.dtype], _TYPES[weight.dtype], rows, cols,
        res["dx"].data_ptr(), res["dweight"].data_ptr(), res["dbias"].data_ptr() if bias else None, _TYPES[dtype],
        int(bool(accumulate)), *_space_args(space), dev.index, _stream(dev.index)))
    if out:
        _written([res[k] for k in out])
    return res


def embedding(ids, weight, scale=1.0, *, vocab_start=0, out=None):
    """Rows scale * weight[ids - vocab_start], of shape ids.shape + (cols,) and weight's type.

    weight holds the rows vocab_start .. vocab_start + len(weight) - 1 of the vocabulary; an id
    outside them (another rank's, or a negative one for padding) gives a row of zeros."""
    start, dev = _int64(vocab_start, "vocab_start"), _gpu(ids, "ids")
    t = _vector(ids, "ids", dev, ids.numel(), _INDEX)
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise _bad("weight must be a matrix")
    vocab, cols, ws = _matrix(weight, "weight", dev, _TYPES)
    shape = ids.shape + (cols,)
    res = weight.new_empty(shape) if out is None else _dense(out, "out", dev, shape, weight.dtype)
    _check(_ops().echo_embedding(t, _INDEX[ids.dtype], weight.data_ptr(), ws, _TYPES[weight.dtype], ids.numel(), cols,
                                 start, vocab, float(scale), res.data_ptr(), dev.index, _stream(dev.index)))
    if out is not None:
        _written(out)
    return res


def embedding_grad(ids, dy, vocab, scale=1.0, *, vocab_start=0, dtype=None, out=None, accumulate=False,
                   workspace=None):
    """Gradient of embedding's table: [vocab, cols], of dy's type or of `dtype` (float32).

    dy has the shape ids.shape + (cols,).  With accumulate=True the rows that ids name are added to `out` and its
    other rows are left alone; otherwise every row is written.  Up to 2^29 tokens, 2^26 rows and 2^42 of their product."""
    start, dev = _int64(vocab_start, "vocab_start"), _gpu(ids, "ids")
    t = _vector(ids, "ids", dev, ids.numel(), _INDEX)
    if not isinstance(dy, torch.Tensor) or dy.dim() != ids.dim() + 1 or dy.shape[:-1] != ids.shape:
        raise _bad("dy must have the shape of ids and one dimension more")
    rows, cols, ds = _matrix(dy, "dy", dev, _TYPES)
    if accumulate and out is None:
        raise _bad("accumulate adds to out")
    if dtype is None:
        dtype = out.dtype if isinstance(out, torch.Tensor) else dy.dtype
    if dtype not in (dy.dtype, torch.float32):
        raise _bad(f"dtype must be {dy.dtype} or torch.float32 (got {dtype})")
    vocab = _int64(vocab, "vocab")
    if vocab < 0:
        raise _bad("vocab must be >= 0")
    res = dy.new_empty((vocab, cols), dtype=dtype) if out is None else _dense(out, "out", dev, (vocab, cols), dtype)
    L = _ops()
    space = _space(workspace, L.echo_embedding_grad_workspace(rows, cols, vocab), dy)
    _check(L.echo_embedding_grad(
        t, _INDEX[ids.dtype], dy.data_ptr(), ds, _TYPES[dy.dtype], rows, cols, start, vocab, float(scale),
        res.data_ptr(), _TYPES[dtype], int(bool(accumulate)), *_space_args(space), dev.index, _stream(dev.index)))
    if out is not None:
        _written(out)
    return res


def _loss_args(logits, targets, vocab_start, vocab_size):
    dev = _gpu(logits, "logits")
    rows, cols, ls = _matrix(logits, "logits", dev, _TYPES)
    if not isinstance(targets, torch.Tensor) or targets.shape != logits.shape[:-1]:
        raise _bad("targets must have the leading shape of logits")
    if vocab_size is None and vocab_start:
        raise _bad("vocab_start needs vocab_size")
    return (dev, rows, cols, ls, _vector(targets, "targets", dev, rows, _INDEX), _int64(vocab_start, "vocab_start"),
            cols if vocab_size is None else _int64(vocab_size, "vocab_size"))


def _grad_out(t, logits, dev, rows, cols):
    """(tensor, row stride) of a gradient of logits: new and dense, or the caller's, of any row stride."""
    if t is None:
        return _like(logits), cols
    n, c, stride = _matrix(t, "grad", dev, (logits.dtype,))
    if t.shape != logits.shape:
        raise _bad(f"grad has shape {tuple(t.shape)}, needs {tuple(logits.shape)}")
    return t, stride


def cross_entropy(logits, targets, *, vocab_start=0, vocab_size=None, grad_loss=None, out=None):
    """Cross entropy of rows of logits; a target outside the vocabulary (-100) marks a row not trained on.

    Whole vocabulary (vocab_size not given): a dict with 'loss' (0 for rows not trained on), 'lse' (log of the sum
    of exponentials), float32, and, if grad_loss (float32, the gradient of each row's loss) is given, 'grad': that of the
    logits, in the same pass.  `out` may supply tensors of those names; 'grad' may be logits itself.

    The rows vocab_start .. vocab_start + cols - 1 of a vocabulary of vocab_size, as one tensor-parallel rank holds
    them: a dict with 'lse' over these rows and 'target', the target's logit or 0 where it is another
    rank's.  The whole lse is the logarithm of the ranks' sum of exp(lse), the target's logit their sum, and
    loss = lse - target; cross_entropy_grad then gives each rank its gradient."""
    dev, rows, cols, ls, t, start, whole = _loss_args(logits, targets, vocab_start, vocab_size)
    shape = logits.shape[:-1]
    if vocab_size is None:
        names = ("loss", "lse")
    else:
        if grad_loss is not None:
            raise _bad("a shard's gradient needs the whole vocabulary's lse: use cross_entropy_grad")
        names = ("lse", "target")
    res = _only(out, names + (("grad",) if grad_loss is not None else ()))
    new = None
    for n in names:
        if n in res:
            res[n] = _dense(res[n], n, dev, shape, torch.float32)
        else:
            res[n] = new = logits.new_empty(shape, dtype=torch.float32) if new is None else torch.empty_like(new)
    g, gs, gl = None, 0, None
    if grad_loss is not None:
        gl = _vector(grad_loss, "grad_loss", dev, rows, (torch.float32,))
        res["grad"], gs = _grad_out(res.get("grad"), logits, dev, rows, cols)
        g = res["grad"].data_ptr()
    _check(_ops().echo_cross_entropy(
        logits.data_ptr(), ls, _TYPES[logits.dtype], t, _INDEX[targets.dtype], rows, cols, start, whole,
        res["lse"].data_ptr(), res["target"].data_ptr() if "target" in res else None,
        res["loss"].data_ptr() if "loss" in res else None, gl, g, gs, dev.index, _stream(dev.index)))
    if out:
        _written([res[k] for k in out])
    return res


def cross_entropy_grad(logits, targets, lse, grad_loss, *, vocab_start=0, vocab_size=None, out=None):
    """(exp(logits - lse) - onehot(targets)) * grad_loss, like logits: the gradient of cross entropy for the
    columns held here, with lse and grad_loss float32 of targets' shape.  `out` may be logits itself."""
    dev, rows, cols, ls, t, start, whole = _loss_args(logits, targets, vocab_start, vocab_size)
    e = _vector(lse, "lse", dev, rows, (torch.float32,))
    gl = _vector(grad_loss, "grad_loss", dev, rows, (torch.float32,))
    res, gs = _grad_out(out, logits, dev, rows, cols)
    _check(_ops().echo_cross_entropy_grad(
        logits.data_ptr(), ls, _TYPES[logits.dtype], t, _INDEX[targets.dtype], rows, cols, start, whole,
        e, gl, res.data_ptr(), gs, dev.index, _stream(dev.index)))
    if out is not None:
        _written(out)
    return res
