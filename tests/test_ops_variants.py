"""The kernels' variants (no GPU): the table that the GPU tests' widths rest on is the sources', and the widths reach all."""
from __future__ import annotations

import os
import re

import pytest

from tests import opsvariants as V

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_12487_amd", "csrc")
RUN = re.compile(r"(?:if \((?:a\.cols|whole) <= (\d+) \* (\d+)\)\s+)?return run\(k_(\w+)<T, \w, (\d+), (\d+), CUT>, (\d+)\);")


def _sources(name):
    """The kernel's variants in the order of the source, with the widest row of each; the last has no bound of its own."""
    found = []
    for file in ("echo_norm.hip", "echo_loss.hip"):
        for a, b, kernel, lanes, each, block in RUN.findall(open(os.path.join(CSRC, file)).read()):
            if kernel == name:
                assert lanes == block
                found.append(((int(lanes), int(each)), int(a) * int(b) if a else None))
    return found


def test_the_table_is_the_sources():
    assert [v for v, _ in _sources("norm")] == V.NORM
    assert [v for v, _ in _sources("loss")] == V.LOSS
    assert [v for v, _ in _sources("norm_grad")] == V.GRAD + V.GRAD_CUT + V.GRAD_WHOLE + [V.GRAD_LAST[2], V.GRAD_LAST[4]]
    for name in ("norm", "loss", "norm_grad"):
        for (lanes, each), bound in _sources(name):
            assert bound in (None, lanes * each)


@pytest.mark.parametrize("rule,widths", [(V.norm, V.NORM_WIDTHS), (V.norm_grad, V.NORM_WIDTHS), (V.loss, V.LOSS_WIDTHS)])
def test_the_widths_reach_every_variant(rule, widths):
    for size in (2, 4):
        every = {rule(c, size) for c in range(1, 70_000)}
        assert len(every) > 14 and every == {rule(c, size) for c in widths}
