"""Argument checks of the training-step operators that need no GPU: sizes and shards out of range."""
from __future__ import annotations

import pytest

from tests.test_ops_abi import E, L, _loss, _loss_grad  # noqa: F401 (fixtures)


@pytest.mark.parametrize("whole", [-1, -2, -(1 << 62), 0, 63])
@pytest.mark.parametrize("call", [_loss, _loss_grad])
def test_a_vocabulary_smaller_than_its_shard_is_refused(E, L, call, whole):
    """A negative size too: with it every target would count as one that is not trained on."""
    kw = dict(loss=None, gl=None, g=None) if call is _loss else {}
    assert call(L, whole=whole, **kw) == E.ECHO_ERR_ARG
    assert "passes the vocabulary" in L.echo_last_error().decode()
