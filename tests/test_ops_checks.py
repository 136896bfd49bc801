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


NOWHERE = 1 << 20      # no such GPU: what passes the checks ends there, with nothing launched
MB = 1 << 20


@pytest.mark.parametrize("what,logits,grad,rows,cols,ls,gs,apart", [
    ("halves of one buffer", 0, 128, 8, 64, 128, 128, True),
    ("halves the other way round", 128, 0, 8, 64, 128, 128, True),
    ("an element into the other half", 0, 126, 8, 64, 128, 128, False),
    ("an element into the next row", 0, 130, 8, 64, 128, 128, False),
    ("the other half, three rows on", 0, 128 + 3 * 256, 8, 64, 128, 128, True),
    ("the same columns, three rows on", 0, 3 * 256, 8, 64, 128, 128, False),
    ("past the last row", 0, 8 * 256, 8, 64, 128, 128, True),
    ("one row in the gap of none", 0, 128, 1, 64, 128, 128, True),
    ("rows that drift through each other's gaps", 0, 128, 8, 64, 128, 192, False),
    ("rows of one repeated", 0, 64, 8, 64, 0, 128, False),
    ("logits whose rows overlap, gradient between their starts", 0, 64, 8, 64, 32, 128, False),
])
def test_only_what_shares_bytes_overlaps(E, L, what, logits, grad, rows, cols, ls, gs, apart):
    """bfloat16 matrices in one buffer, offsets in bytes."""
    rc = L.echo_cross_entropy_grad(MB + logits, ls, 2, 3 * MB, 1, rows, cols, 0, cols, 4 * MB, 5 * MB, MB + grad, gs, NOWHERE, None)
    assert rc == (E.ECHO_ERR_HIP if apart else E.ECHO_ERR_ARG), (what, L.echo_last_error())
    assert apart or "grad overlaps logits" in L.echo_last_error().decode()


def test_a_vector_between_the_rows_of_a_matrix(E, L):
    def call(lse, rows=8):
        return L.echo_cross_entropy(MB, 128, 2, 3 * MB, 1, rows, 64, 0, 64, lse, None, 5 * MB, None, None, 0, NOWHERE, None)

    assert call(MB + 128) == E.ECHO_ERR_HIP                   # 32 bytes in the first row's gap
    assert call(MB + 128, rows=1) == E.ECHO_ERR_HIP
    assert call(MB + 256 - 16) == E.ECHO_ERR_ARG              # into the second row
    assert call(MB + 64) == E.ECHO_ERR_ARG


def test_shard_starts_beyond_64_bits_are_refused(E, monkeypatch):
    """ctypes would cut them to 64 bits: 2^64 would be the id 0."""
    for n in (1 << 63, 1 << 64, -(1 << 63) - 1, 1 - (1 << 64)):
        with pytest.raises(E.EchoError, match="64 bits") as e:
            E.ops._int64(n, "vocab_start")
        assert e.value.code == E.ECHO_ERR_ARG
    for n in (0, 5, (1 << 63) - 1, -(1 << 63)):
        assert E.ops._int64(n, "vocab_start") == n
