"""Argument checks of the training-step operators that need no GPU: sizes and shards out of range."""
from __future__ import annotations

import pytest

from tests.test_ops_abi import E, L, _embed_grad, _loss, _loss_grad  # noqa: F401 (fixtures)


@pytest.mark.parametrize("whole", [-1, -2, -(1 << 62), 0, 63])
@pytest.mark.parametrize("call", [_loss, _loss_grad])
def test_a_vocabulary_smaller_than_its_shard_is_refused(E, L, call, whole):
    """A negative size too: with it every target would count as one that is not trained on."""
    kw = dict(loss=None, gl=None, g=None) if call is _loss else {}
    assert call(L, whole=whole, **kw) == E.ECHO_ERR_ARG
    assert "passes the vocabulary" in L.echo_last_error().decode()


def test_a_sort_of_unbounded_work_is_out_of_range(E, L):
    """The ids are looked through by every sorting workgroup, vocab / 64 of them: 2^29 tokens and 2^26 rows, each allowed
    by itself, would take minutes in one launch.  (At the bound the calls here go on to the workspace's check.)"""
    for rows, vocab in ((1 << 20, 1 << 22), (1 << 29, 1 << 13), (1 << 16, 1 << 26)):
        assert _embed_grad(L, rows=rows, cols=1, vocab=vocab, ws=None) == E.ECHO_ERR_ARG
        assert "workspace" in L.echo_last_error().decode()
    for rows, vocab in (((1 << 20) + 1, 1 << 22), (1 << 20, (1 << 22) + 1), (1 << 29, 1 << 26)):
        assert _embed_grad(L, rows=rows, cols=1, vocab=vocab, ws=None) == E.ECHO_ERR_RANGE
        assert "2^42" in L.echo_last_error().decode()


class _Function:
    """A library function that keeps every result type it was ever given."""

    def __init__(self):
        self.__dict__["types"] = []

    def __setattr__(self, name, value):
        if name == "restype":
            self.types.append(value)
        self.__dict__[name] = value


class _Library:
    def __getattr__(self, name):
        self.__dict__[name] = _Function()
        return self.__dict__[name]


def test_signatures_hold_while_another_thread_sets_them(E, monkeypatch):
    """Two threads may both come first.  The second sets what the first may already be calling, so no function has
    another signature in between: a workspace size cut to 32 bits would be too small a workspace."""
    import ctypes

    fake = _Library()
    monkeypatch.setattr(E.ops, "lib", lambda: fake)
    monkeypatch.setattr(E.ops, "_fns", None)
    assert E.ops._ops() is fake
    for name in E.ops.EXPORTS:
        size = name.endswith("_workspace")
        assert getattr(fake, name).types == [ctypes.c_int64 if size else ctypes.c_int32], name
        assert getattr(fake, name).argtypes
