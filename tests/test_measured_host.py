"""Durations of a graph's operators given from outside (no GPU): which ops take them."""
from __future__ import annotations

import numpy as np
import pytest

from workloads import configs, gpt1f1b


def test_given_durations_replace_only_their_operators():
    base = configs.graph(1)
    p = configs.graph_params(1)
    ranks = p["tp"] * p["dp"]                       # of one pipeline stage
    layers, m = p["n_layers"], p["microbatches"]
    # two norms a layer and the last one; the embedding on the first stage, the loss on the last
    count = {"embed": m * ranks, "norm": m * ranks * (2 * layers + 1), "loss": m * ranks, "loss_grad": m * ranks,
             "norm_grad": m * ranks * (2 * layers + 1), "embed_grad": m * ranks}
    assert set(count) == set(gpt1f1b.OPERATORS)
    used = np.zeros(len(base["op_dur"]), bool)
    for name in gpt1f1b.OPERATORS:
        g = configs.graph(1, operator_ns={name: 123})
        changed = g["op_dur"] != base["op_dur"]
        assert int(changed.sum()) == count[name] and (g["op_dur"][changed] == 123).all()
        assert (g["op_kind"][changed] == gpt1f1b.KIND_COMPUTE).all() and not (used & changed).any()
        used |= changed
        assert set(g) == set(base)
        for k in g:
            if k != "op_dur":
                assert np.array_equal(g[k], base[k]), k


def test_durations_are_at_least_one_and_names_are_checked():
    g = configs.graph(1, operator_ns={"norm": 0})
    assert (g["op_dur"] == 1).sum() > 0
    with pytest.raises(ValueError, match="unknown operators"):
        configs.graph(1, operator_ns={"gemm": 5})
    assert np.array_equal(configs.graph(1, operator_ns={})["op_dur"], configs.graph(1)["op_dur"])
