"""C-ABI checks of the training-step operators that need no GPU: exported symbols, workspace sizes, and the
refusals, which all come before the device is touched (the pointers here point at nothing)."""
from __future__ import annotations

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, I64 = 0, 1, 2, 1


@pytest.fixture(scope="module")
def E():
    import paper_2412_12487_amd as E
    if not os.path.exists(E.LIB_PATH):
        from paper_2412_12487_amd import build
        build.build()
    return E


@pytest.fixture(scope="module")
def L(E):
    return E.ops._ops()


def test_library_exports_every_declared_operator(E, L):
    header = open(os.path.join(ROOT, "include", "echo_ops.h")).read()
    declared = set(re.findall(r"\b(echo_[a-z_]+)\s*\(", header))
    assert declared == set(E.ops.EXPORTS)
    assert all(hasattr(L, name) for name in declared)
    assert all(n in E.__all__ and callable(getattr(E, n)) for n in ("layer_norm", "embedding_grad", "cross_entropy"))
    with pytest.raises(AttributeError):
        E.no_such_operator


def test_binding_refuses_tensors_off_the_gpu(E):
    import torch
    x = torch.zeros(2, 8)
    for call in (lambda: E.layer_norm(x, x[0], x[0]), lambda: E.embedding(torch.zeros(2, dtype=torch.int64), x),
                 lambda: E.cross_entropy(x, torch.zeros(2, dtype=torch.int64))):
        with pytest.raises(E.EchoError, match="GPU"):
            call()


MB = 1 << 20      # buffers of the calls below, a megabyte apart


def _norm(L, **k):
    a = dict(x=MB, xs=64, r=None, rs=0, w=3 * MB, b=4 * MB, type=BF16, wt=BF16, rows=8, cols=64, eps=1e-5, y=5 * MB, sum=None,
             mean=7 * MB, rstd=8 * MB)
    a.update(k)
    return L.echo_layer_norm(*a.values(), 0, None)


def _norm_grad(L, **k):
    a = dict(dy=MB, ds=64, x=2 * MB, xs=64, w=3 * MB, mean=4 * MB, rstd=5 * MB, r=None, rs=0, type=BF16, wt=BF16, rows=8, cols=64,
             dx=7 * MB, dw=8 * MB, db=9 * MB, gt=F32, acc=0, ws=10 * MB, wb=MB)
    a.update(k)
    return L.echo_layer_norm_grad(*a.values(), 0, None)


def _embed(L, **k):
    a = dict(ids=MB, it=I64, w=2 * MB, ws=64, type=BF16, rows=8, cols=64, start=0, vocab=100, scale=1.0, out=4 * MB)
    a.update(k)
    return L.echo_embedding(*a.values(), 0, None)


def _embed_grad(L, **k):
    a = dict(ids=MB, it=I64, dy=2 * MB, ds=64, type=BF16, rows=8, cols=64, start=0, vocab=100, scale=1.0, dw=4 * MB, gt=BF16,
             acc=0, ws=10 * MB, wb=4 * MB)
    a.update(k)
    return L.echo_embedding_grad(*a.values(), 0, None)


def _loss(L, **k):
    a = dict(l=MB, ls=64, type=BF16, t=2 * MB, it=I64, rows=8, cols=64, start=0, whole=64, lse=3 * MB, target=None, loss=4 * MB,
             gl=5 * MB, g=6 * MB, gs=64)
    a.update(k)
    return L.echo_cross_entropy(*a.values(), 0, None)


def _loss_grad(L, **k):
    a = dict(l=MB, ls=64, type=BF16, t=2 * MB, it=I64, rows=8, cols=64, start=0, whole=64, lse=3 * MB, gl=5 * MB, g=6 * MB, gs=64)
    a.update(k)
    return L.echo_cross_entropy_grad(*a.values(), 0, None)


REFUSED = [
    (_norm, dict(x=None), "x is null"), (_norm, dict(y=None), "y is null"), (_norm, dict(w=None), "weight is null"),
    (_norm, dict(mean=None), "mean is null"), (_norm, dict(type=3), "unknown element type"),
    (_norm, dict(wt=F16), "weight_type"), (_norm, dict(rows=-1), "rows"), (_norm, dict(rows=1 << 31), "rows"),
    (_norm, dict(cols=0), "cols"), (_norm, dict(cols=(1 << 24) + 1), "cols"), (_norm, dict(xs=-64), "stride"),
    (_norm, dict(xs=1 << 40), "stride"), (_norm, dict(eps=-1.0), "eps"), (_norm, dict(eps=float("inf")), "eps"),
    (_norm, dict(x=MB + 1), "aligned"), (_norm, dict(mean=7 * MB + 2), "aligned"), (_norm, dict(r=6 * MB, rs=64), "sum"),
    (_norm, dict(sum=6 * MB), "sum"), (_norm, dict(y=MB), "overlaps x"), (_norm, dict(y=MB + 1022), "overlaps x"),
    (_norm, dict(mean=5 * MB), "overlap"), (_norm, dict(r=6 * MB, rs=64, sum=MB, xs=65), "overlaps x"),
    (_norm_grad, dict(dy=None), "dy is null"), (_norm_grad, dict(dw=None), "dweight is null"),
    (_norm_grad, dict(gt=F16), "grad_type"), (_norm_grad, dict(wt=F32, gt=BF16), "grad_type"),
    (_norm_grad, dict(ws=None), "workspace"), (_norm_grad, dict(wb=4), "workspace"),
    (_norm_grad, dict(ws=10 * MB + 8), "workspace is not aligned"), (_norm_grad, dict(dx=2 * MB), "overlaps x"),
    (_norm_grad, dict(dx=MB, ds=66), "overlaps dy"), (_norm_grad, dict(dw=9 * MB), "overlap"),
    (_norm_grad, dict(ws=MB), "workspace overlaps dy"),
    (_embed, dict(ids=None), "ids is null"), (_embed, dict(it=2), "index type"), (_embed, dict(start=-1), "shard"),
    (_embed, dict(vocab=-1), "shard"), (_embed, dict(vocab=1 << 31), "shard"), (_embed, dict(start=(1 << 63) - 1), "shard"),
    (_embed, dict(ids=MB + 4), "aligned"), (_embed, dict(out=2 * MB), "overlaps weight"), (_embed, dict(w=None), "weight is null"),
    (_embed_grad, dict(dw=None), "dweight is null"), (_embed_grad, dict(gt=F16), "grad_type"),
    (_embed_grad, dict(wb=16), "workspace"), (_embed_grad, dict(dw=2 * MB), "overlaps dy"),
    (_embed_grad, dict(dw=10 * MB), "overlap"),
    (_loss, dict(whole=63), "passes the vocabulary"), (_loss, dict(whole=65), "whole vocabulary"),
    (_loss, dict(gl=None), "grad_loss"), (_loss, dict(g=None), "grad_loss"), (_loss, dict(gs=63), "rows of grad"),
    (_loss, dict(lse=None, loss=None, gl=None, g=None), "no output"), (_loss, dict(g=MB, ls=66), "overlaps logits"),
    (_loss, dict(lse=4 * MB), "overlap"), (_loss, dict(t=None), "targets is null"),
    (_loss_grad, dict(lse=None), "lse is null"), (_loss_grad, dict(g=None), "grad is null"), (_loss_grad, dict(gs=0), "rows of grad"),
    (_loss_grad, dict(g=MB + 128), "overlaps logits"), (_loss_grad, dict(whole=10), "passes the vocabulary"),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals_come_before_the_device(E, L, i):
    call, change, msg = REFUSED[i]
    assert call(L, **change) == E.ECHO_ERR_ARG
    assert msg in L.echo_last_error().decode()


def test_more_elements_than_a_grid_holds_are_out_of_range(E, L):
    for call in (_norm, _norm_grad, _embed, _embed_grad, _loss_grad):
        kw = {} if call is not _loss_grad else dict(whole=1 << 20)
        assert call(L, rows=(1 << 18) + 1, cols=1 << 20, **kw) == E.ECHO_ERR_RANGE
    assert _embed_grad(L, vocab=(1 << 26) + 1) == E.ECHO_ERR_RANGE


def test_calls_without_work_succeed_and_clear_the_error(E, L):
    assert _norm(L, cols=0) == E.ECHO_ERR_ARG and L.echo_last_error()
    assert _norm(L, rows=0, x=None, y=None, w=None, b=None, mean=None, rstd=None) == E.ECHO_OK
    assert L.echo_last_error() == b""
    assert _embed(L, rows=0, ids=None, out=None) == E.ECHO_OK
    assert _embed_grad(L, vocab=0, dw=None) == E.ECHO_OK
    assert _embed_grad(L, rows=0, acc=1, ids=None, dy=None, ws=None, wb=0) == E.ECHO_OK
    assert _loss(L, rows=0, l=None, t=None) == E.ECHO_OK
    assert _loss_grad(L, rows=0, l=None, t=None, lse=None, gl=None, g=None) == E.ECHO_OK


def test_workspace_sizes(L):
    """Positive where there is work, 0 outside the documented sizes, and no overflow at the largest."""
    norm, embed = L.echo_layer_norm_grad_workspace, L.echo_embedding_grad_workspace
    assert norm(-1, 8) == norm(8, 0) == embed(8, 0, 8) == embed(-1, 8, 8) == embed(8, 8, -1) == embed(0, 8, 8) == 0
    assert norm(8, 64) >= 8 * 64 and embed(8, 64, 100) >= 4 * 108
    assert 0 < norm((1 << 31) - 1, 1 << 24) < 1 << 50
    assert 0 < embed((1 << 31) - 1, 1 << 24, 1 << 26) < 1 << 56 and embed(8, 8, (1 << 26) + 1) == 0
    assert ctypes.sizeof(ctypes.c_int64) == 8


def test_more_tokens_than_a_sort_takes_are_out_of_range(E, L):
    assert _embed_grad(L, rows=(1 << 29) + 1, cols=1) == E.ECHO_ERR_RANGE
    assert "2^29" in L.echo_last_error().decode()
