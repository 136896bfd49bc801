"""Edges of the training-step operators: statistics at the edge of 32 bits, arguments between each other's rows."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2412_12487_amd as E
from tests import opsref as R

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, mean=0.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


# rows that leave lanes of their team idle, whole pieces and cut ones, from the narrowest team to past the widest
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [5, 104, 101, 904, 1001, 1600, 1501, 3200, 3001, 5600, 5003, 7200, 7001, 10400, 10001, 15200, 15001,
                                  20003])
def test_layer_norm_grad_where_mean_times_rstd_passes_32_bits(cols, dtype):
    """A constant row of 2^120 has finite statistics, and n = 0 throughout: its gradient is rstd * (g - mean(g)), although
    2^120 / sqrt(1e-5 * 2^-20) is no 32-bit number."""
    g = _gen(cols)
    x, w = _normal(g, 5, cols, dtype=dtype), _normal(g, cols, std=0.2, mean=1.0, dtype=dtype)
    dy, dr = _normal(g, 5, cols, std=0.5, dtype=dtype), _normal(g, 5, cols, dtype=dtype)
    s = E.layer_norm(x, w, None)
    x[2], s["mean"][2], s["rstd"][2] = 2.0 ** 120, 2.0 ** 120, 1024 / math.sqrt(1e-5)
    assert math.isinf(float(s["mean"][2] * s["rstd"][2]))
    out = E.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], grad_residual=dr, dtype=F32)
    for k, (v, e) in R.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], dr).items():
        R.close(out[k], v, e, k)


@pytest.mark.parametrize("cols", [3, 64, 517, 2056, 20001, 70001])
def test_cross_entropy_gradient_between_the_rows_of_the_logits(cols):
    """Column halves of one buffer: nothing shares a byte, and nothing outside the gradient's half is written."""
    g = _gen(cols)
    pad = 5
    buf = _normal(g, 9, 2 * cols + pad, std=2.0, dtype=BF16)
    t = torch.randint(0, cols, (9,), generator=g, device="cuda")
    gl = _normal(g, 9)
    for lo, hi in ((0, cols + pad), (cols + pad, 0)):
        before = buf.clone()
        l, d = buf[:, lo:lo + cols], buf[:, hi:hi + cols]
        want = E.cross_entropy(l.clone(), t, grad_loss=gl)
        got = E.cross_entropy(l, t, grad_loss=gl, out={"grad": d})
        assert all(torch.equal(got[k], want[k]) for k in want)
        d.copy_(before[:, hi:hi + cols])
        got = E.cross_entropy_grad(l, t, want["lse"], gl, out=d)
        assert torch.equal(got, E.cross_entropy_grad(l.clone(), t, want["lse"], gl))
        d.copy_(before[:, hi:hi + cols])
        assert torch.equal(buf, before)


@pytest.mark.parametrize("start", [1 << 63, 1 << 64, 1 - (1 << 64)])
def test_shards_that_start_beyond_64_bits_are_refused(start):
    table, logits = torch.ones(10, 4, device="cuda"), torch.zeros(2, 8, device="cuda")
    ids = torch.tensor([0, 3], device="cuda")
    for call in (lambda: E.embedding(ids, table, vocab_start=start),
                 lambda: E.embedding_grad(ids, table[:2], 10, vocab_start=start),
                 lambda: E.cross_entropy(logits, ids, vocab_start=start, vocab_size=100),
                 lambda: E.cross_entropy(logits, ids, vocab_start=0, vocab_size=start),
                 lambda: E.cross_entropy_grad(logits, ids, logits[:, 0].contiguous(), logits[:, 1].contiguous(), vocab_start=start,
                                              vocab_size=100)):
        with pytest.raises(E.EchoError, match="64 bits"):
            call()


def _calls():
    """{name: (call of the tensors, those tensors)} over every input and every tensor that may be written."""
    g = _gen(7)
    x, r, dy = (_normal(g, 6, 40) for _ in range(3))
    w, b = _normal(g, 40), _normal(g, 40)
    s = E.layer_norm(x, w, b)
    ids, table = torch.arange(6, device="cuda"), _normal(g, 9, 40)
    logits, gl, lse = _normal(g, 6, 40), _normal(g, 6), _normal(g, 6)
    e = torch.empty_like
    return {
        "layer_norm": (lambda x, w, b, r, y, t: E.layer_norm(x, w, b, residual=r, out={"y": y, "sum": t}), (x, w, b, r, e(x), e(x)), 4),
        "layer_norm_grad": (lambda dy, x, w, m, k, r, dx, dw, db: E.layer_norm_grad(
            dy, x, w, m, k, grad_residual=r, out={"dx": dx, "dweight": dw, "dbias": db}),
            (dy, x, w, s["mean"], s["rstd"], r, e(x), e(w), e(b)), 6),
        "embedding": (lambda w, o: E.embedding(ids, w, out=o), (table, e(x)), 1),
        "embedding_grad": (lambda dy, o: E.embedding_grad(ids, dy, 9, out=o), (dy, e(table)), 1),
        "cross_entropy": (lambda l, gl, d, lse: E.cross_entropy(l, ids, grad_loss=gl, out={"grad": d, "lse": lse}),
                          (logits, gl, e(logits), e(gl)), 2),
        "cross_entropy_grad": (lambda l, lse, gl, d: E.cross_entropy_grad(l, ids, lse, gl, out=d), (logits, lse, gl, e(logits)), 3),
    }


@pytest.mark.parametrize("name", ["layer_norm", "layer_norm_grad", "embedding", "embedding_grad", "cross_entropy", "cross_entropy_grad"])
def test_tensors_that_require_grad_are_refused_where_a_graph_is_recorded(name):
    """The calls record nothing for automatic differentiation: a gradient would be lost without a word."""
    call, tensors, _ = _calls()[name]
    call(*tensors)
    for i in range(len(tensors)):
        leaf = [t.clone().requires_grad_(k == i) for k, t in enumerate(tensors)]
        with pytest.raises(E.EchoError, match="requires grad"):
            call(*leaf)
        with torch.no_grad():
            call(*leaf)
        call(*[t.detach() for t in leaf])


@pytest.mark.parametrize("name", ["layer_norm", "layer_norm_grad", "embedding", "embedding_grad", "cross_entropy", "cross_entropy_grad"])
def test_a_saved_tensor_that_a_call_wrote_is_noticed(name):
    """As after any in-place operation: backward through a tensor that was written since raises."""
    call, tensors, first = _calls()[name]
    for i in range(first, len(tensors)):
        leaf = torch.zeros_like(tensors[i]).requires_grad_()
        saved = leaf.exp()                 # its backward reads what it returned
        call(*[saved.detach() if k == i else t for k, t in enumerate(tensors)])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            saved.sum().backward()
    kept = torch.zeros_like(tensors[0]).requires_grad_()
    read = kept.exp()
    call(read.detach(), *tensors[1:])      # an input is only read
    read.sum().backward()


def test_outputs_over_inputs_count_as_written():
    g = _gen(8)
    x, r, w = _normal(g, 6, 40), _normal(g, 6, 40), _normal(g, 40)
    ids, gl = torch.arange(6, device="cuda"), _normal(g, 6)
    s = E.layer_norm(x, w)
    for call in (lambda t: E.layer_norm(t, w, residual=r, out={"sum": t}), lambda t: E.layer_norm(x, w, residual=t, out={"sum": t}),
                 lambda t: E.layer_norm_grad(t, x, w, s["mean"], s["rstd"], out={"dx": t}),
                 lambda t: E.cross_entropy(t, ids, grad_loss=gl, out={"grad": t}),
                 lambda t: E.cross_entropy_grad(t, ids, gl, gl, out=t)):
        saved = _normal(g, 6, 40).requires_grad_().exp()
        call(saved.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            saved.sum().backward()


@pytest.mark.parametrize("cols", [3, 50, 4096, 51200, 70000])
def test_statistics_of_rows_with_nan_or_infinity(cols):
    """No sum of exponentials has a value there: lse and loss are NaN; the target's logit is what it is."""
    l = _normal(_gen(cols), 5, cols, dtype=BF16)
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    l[1, cols - 1], l[2, cols - 1], l[3, cols // 2], l[3, cols - 1] = math.nan, math.inf, math.nan, math.inf
    out = E.cross_entropy(l, t)
    bad = torch.tensor([False, True, True, True, False], device="cuda")
    assert torch.equal(torch.isnan(out["lse"]), bad) and torch.equal(torch.isnan(out["loss"]), bad)
    part = E.cross_entropy(l, t, vocab_start=0, vocab_size=cols + 9)
    assert torch.equal(torch.isnan(part["lse"]), bad) and torch.equal(part["target"], l[:, 0].float())
