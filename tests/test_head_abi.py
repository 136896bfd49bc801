"""C-ABI and binding checks of distillation and of the output head's losses that need no GPU: workspace sizes and refusals, which
all come before the device is touched (the pointers here point at nothing)."""
from __future__ import annotations

import pytest

from tests.test_ops_abi import E, L  # noqa: F401 (fixtures)

F32, F16, BF16, I32, I64 = 0, 1, 2, 0, 1
MB = 1 << 20
NOWHERE = 1 << 20      # no such GPU: what passes the checks ends there, with nothing launched


def _distill(L, **k):
    a = dict(l=MB, ls=64, type=BF16, ids=2 * MB, it=I64, z=3 * MB, zt=F32, rows=8, cols=64, top=4, start=0, whole=64, temp=2.0,
             lse=4 * MB, target=None, entropy=None, loss=5 * MB, gl=6 * MB, g=7 * MB, gs=64)
    a.update(k)
    return L.echo_distillation(*a.values(), NOWHERE, None)


def _distill_grad(L, **k):
    a = dict(l=MB, ls=64, type=BF16, ids=2 * MB, it=I64, z=3 * MB, zt=F32, rows=8, cols=64, top=4, start=0, whole=64, temp=2.0,
             lse=4 * MB, gl=6 * MB, g=7 * MB, gs=64)
    a.update(k)
    return L.echo_distillation_grad(*a.values(), NOWHERE, None)


def _linear(L, **k):
    a = dict(h=MB, hs=64, w=2 * MB, ws=64, type=BF16, t=3 * MB, it=I64, rows=8, cols=64, vocab=100, start=0, whole=100, lse=4 * MB,
             target=None, loss=5 * MB, gl=6 * MB, dh=7 * MB, dw=8 * MB, gt=BF16, acc=0, space=16 * MB, bytes=64 * MB)
    a.update(k)
    return L.echo_linear_cross_entropy(*a.values(), NOWHERE, None)


def _linear_grad(L, **k):
    a = dict(h=MB, hs=64, w=2 * MB, ws=64, type=BF16, t=3 * MB, it=I64, rows=8, cols=64, vocab=100, start=0, whole=100, lse=4 * MB,
             gl=6 * MB, dh=7 * MB, dw=8 * MB, gt=BF16, acc=0, space=16 * MB, bytes=64 * MB)
    a.update(k)
    return L.echo_linear_cross_entropy_grad(*a.values(), NOWHERE, None)


def _lindist(L, **k):
    a = dict(h=MB, hs=64, w=2 * MB, ws=64, type=BF16, ids=3 * MB, it=I64, z=9 * MB, zt=F32, rows=8, cols=64, vocab=100, top=4, start=0,
             whole=100, temp=2.0, lse=4 * MB, target=None, entropy=None, loss=5 * MB, gl=6 * MB, dh=7 * MB, dw=8 * MB, gt=BF16, acc=0,
             space=16 * MB, bytes=64 * MB)
    a.update(k)
    return L.echo_linear_distillation(*a.values(), NOWHERE, None)


def _lindist_grad(L, **k):
    a = dict(h=MB, hs=64, w=2 * MB, ws=64, type=BF16, ids=3 * MB, it=I64, z=9 * MB, zt=F32, rows=8, cols=64, vocab=100, top=4, start=0,
             whole=100, temp=2.0, lse=4 * MB, gl=6 * MB, dh=7 * MB, dw=8 * MB, gt=BF16, acc=0, space=16 * MB, bytes=64 * MB)
    a.update(k)
    return L.echo_linear_distillation_grad(*a.values(), NOWHERE, None)


CALLS = [_distill, _distill_grad, _linear, _linear_grad, _lindist, _lindist_grad]
TEACHERS = [_distill, _distill_grad, _lindist, _lindist_grad]
HEADS = [_linear, _linear_grad, _lindist, _lindist_grad]


def _refused(E, L, rc, code, text):
    assert rc == code, L.echo_last_error()
    assert text in L.echo_last_error().decode()


@pytest.mark.parametrize("call", CALLS)
def test_good_arguments_reach_the_device(E, L, call):
    assert call(L) == E.ECHO_ERR_HIP
    assert call(L, it=I32) == E.ECHO_ERR_HIP
    assert call(L, start=3, whole=1 << 40, **(dict(loss=None, gl=None, **(dict(g=None) if call is _distill else dict(dh=None, dw=None)))
                                               if call in (_distill, _linear, _lindist) else {})) == E.ECHO_ERR_HIP


@pytest.mark.parametrize("call", CALLS)
def test_common_refusals(E, L, call):
    bad = E.ECHO_ERR_ARG
    _refused(E, L, call(L, type=3), bad, "element type")
    _refused(E, L, call(L, it=2), bad, "index type")
    _refused(E, L, call(L, rows=-1), bad, "rows")
    _refused(E, L, call(L, cols=0), bad, "cols")
    _refused(E, L, call(L, whole=10), bad, "passes the vocabulary")
    _refused(E, L, call(L, start=-1), bad, "out of range")
    _refused(E, L, call(L, start=1), bad, "passes the vocabulary")
    _refused(E, L, call(L, gl=6 * MB + 2), bad, "aligned")
    _refused(E, L, call(L, gl=None), bad, "grad_loss")
    first = "l" if call in (_distill, _distill_grad) else "h"
    _refused(E, L, call(L, **{first: None}), bad, "is null")
    _refused(E, L, call(L, **{first: MB + 1}), bad, "aligned")
    _refused(E, L, call(L, **{first + "s": -1}), bad, "stride")
    _refused(E, L, call(L, **{first + "s": (1 << 28) + 1}), bad, "stride")


@pytest.mark.parametrize("call", TEACHERS)
def test_teachers_refusals(E, L, call):
    bad = E.ECHO_ERR_ARG
    for top in (0, -1, 1025):
        _refused(E, L, call(L, top=top), bad, "top")
    for temp in (0.0, -1.0, float("nan"), float("inf"), 1e-7, 1e7):
        _refused(E, L, call(L, temp=temp), bad, "temperature")
    _refused(E, L, call(L, zt=F16), bad, "teacher_type")
    _refused(E, L, call(L, type=F32, zt=BF16), bad, "teacher_type")
    _refused(E, L, call(L, ids=None), bad, "ids is null")
    _refused(E, L, call(L, z=None), bad, "teacher is null")
    assert call(L, top=1024, temp=1e6, **({} if call in (_distill, _distill_grad) else dict(bytes=1 << 40))) == E.ECHO_ERR_HIP


@pytest.mark.parametrize("call", [_distill, _linear, _lindist])
def test_losses_of_a_shard_and_outputs(E, L, call):
    bad = E.ECHO_ERR_ARG
    _refused(E, L, call(L, whole=1000), bad, "shard")
    grads = dict(g=None) if call is _distill else dict(dh=None, dw=None)
    _refused(E, L, call(L, loss=None, lse=None, gl=None, **grads), bad, "no output")
    _refused(E, L, call(L, **grads), bad, "grad_loss")
    assert call(L, gl=None, **grads) == E.ECHO_ERR_HIP
    if call is not _distill:
        _refused(E, L, call(L, dh=None), bad, "together")
        _refused(E, L, call(L, lse=None), bad, "lse")
    assert call(L, rows=0) in (E.ECHO_OK, E.ECHO_ERR_HIP)      # the table's gradient is zeros


@pytest.mark.parametrize("call", HEADS)
def test_heads_refusals(E, L, call):
    bad, out = E.ECHO_ERR_ARG, E.ECHO_ERR_RANGE
    _refused(E, L, call(L, w=None), bad, "weight is null")
    _refused(E, L, call(L, vocab=0, whole=0), bad, "vocab")
    _refused(E, L, call(L, vocab=(1 << 24) + 1, whole=1 << 25), bad, "vocab")
    _refused(E, L, call(L, rows=(1 << 24) + 1), bad, "rows")
    _refused(E, L, call(L, cols=(1 << 20) + 1), bad, "cols")
    _refused(E, L, call(L, rows=1 << 20, vocab=1 << 20, whole=1 << 20), out, "2^38")
    _refused(E, L, call(L, gt=F16), bad, "grad_type")
    _refused(E, L, call(L, space=None), bad, "workspace")
    _refused(E, L, call(L, bytes=16), bad, "workspace")
    _refused(E, L, call(L, space=16 * MB + 8), bad, "workspace")
    _refused(E, L, call(L, dh=MB), bad, "dhidden overlaps hidden")
    _refused(E, L, call(L, dw=2 * MB), bad, "dweight overlaps weight")
    _refused(E, L, call(L, dw=7 * MB), bad, "overlap")
    _refused(E, L, call(L, dw=16 * MB), bad, "overlap")
    assert call(L, gt=F32) == E.ECHO_ERR_HIP


@pytest.mark.parametrize("call", [_distill, _distill_grad])
def test_a_gradient_may_be_the_logits(E, L, call):
    bad = E.ECHO_ERR_ARG
    assert call(L, g=MB) == E.ECHO_ERR_HIP
    _refused(E, L, call(L, g=MB + 2), bad, "grad overlaps logits")
    _refused(E, L, call(L, g=3 * MB), bad, "grad overlaps teacher")
    _refused(E, L, call(L, gs=63), bad, "rows of grad overlap")


def test_workspaces(E, L):
    def need(h=MB, hs=64, w=2 * MB, ws=64, type=BF16, rows=8, cols=64, vocab=100, top=0, loss=1, grads=1):
        return L.echo_linear_workspace(h, hs, w, ws, type, rows, cols, vocab, top, loss, grads)

    assert need(rows=0) == need(type=7) == need(vocab=0) == need(cols=0) == need(top=1025) == 0
    base = need()
    assert 0 < need(grads=0) < base
    copied = need(h=MB + 2)
    assert copied >= base + 8 * 64 * 2                      # rows at odd places are laid out first
    assert need(cols=63, hs=63, ws=63) > need(grads=1)
    assert need(type=F32) > 2 * base
    # the gradient's shares are held a gigabyte at a time, whatever the sizes
    big = need(rows=1 << 16, cols=1024, hs=1024, ws=1024, vocab=50000)
    assert (1 << 30) * 0.9 < big < (1 << 30) + (1 << 16) * 1024 * 4 + (1 << 28)


def test_binding_refuses(E):
    import torch

    x, t, g = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    ids = torch.zeros(2, 3, dtype=torch.int64)
    for call in (lambda: E.linear_cross_entropy(x, x, t), lambda: E.linear_cross_entropy_grad(x, x, t, g, g),
                 lambda: E.distillation(x, ids, ids.float()), lambda: E.distillation_grad(x, ids, ids.float(), g, g),
                 lambda: E.linear_distillation(x, x, ids, ids.float()),
                 lambda: E.linear_distillation_grad(x, x, ids, ids.float(), g, g)):
        with pytest.raises(E.EchoError, match="GPU"):
            call()
