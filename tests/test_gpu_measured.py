"""The training step's operators run together, and the durations measured for a graph."""
from __future__ import annotations

import pytest
import torch
import torch.nn.functional as F

import paper_2412_12487_amd as E
from workloads import configs, gpt1f1b, measured

pytestmark = pytest.mark.gpu


def _model(dtype, tokens=70, vocab=90, hidden=48, blocks=3):
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets[3] = -100
    norms = [((1 + 0.2 * r(hidden)).to(dtype), (0.2 * r(hidden)).to(dtype)) for _ in range(blocks)]
    return ids, targets, (0.3 * r(vocab, hidden)).to(dtype), norms


def _exact(ids, targets, table, norms, scale, eps):
    """The same pass in 64 bits by automatic differentiation, on the CPU."""
    leaf = lambda t: t.cpu().double().requires_grad_()
    table, norms = leaf(table), [(leaf(w), leaf(b)) for w, b in norms]
    h = table[ids.cpu()] * scale
    for k, (w, b) in enumerate(norms):
        y = F.layer_norm(h, h.shape[-1:], w, b, eps)
        if k + 1 < len(norms):
            h = h + y
    loss = F.cross_entropy(y @ table.t(), targets.cpu(), ignore_index=-100)
    loss.backward()
    return loss.detach(), table.grad, [(w.grad, b.grad) for w, b in norms]


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 0.05)])
def test_training_step_against_automatic_differentiation(dtype, tol):
    """float32: under 200 roundings of 2^-24 along any path, 1.2e-5 of the norm if all went one way; they do not.
    bfloat16: about ten roundings of 2^-9 along a path (activations, logits and gradients), with room for the
    norms' gain (rstd is about 1.5 here)."""
    ids, targets, table, norms = _model(dtype)
    out = measured.training_step(ids, targets, table, norms, scale=2.0)
    loss, dtable, dnorms = _exact(ids, targets, table, norms, 2.0, 1e-5)
    assert abs(float(out["loss"]) - float(loss)) <= tol * float(loss)
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    assert out["table"].dtype == torch.float32 and off(out["table"], dtable) <= tol
    for (dw, db), (ew, eb) in zip(out["norms"], dnorms):
        assert off(dw, ew) <= tol and off(db, eb) <= tol


def test_training_learns():
    ids, targets, table, norms = _model(torch.float32)
    losses = []
    for _ in range(30):
        out = measured.training_step(ids, targets, table, norms)
        losses.append(out["loss"])
        table -= 0.5 * out["table"]
        for (w, b), (dw, db) in zip(norms, out["norms"]):
            w -= 0.5 * dw
            b -= 0.5 * db
    losses = torch.stack(losses).tolist()
    assert losses[-1] < 0.7 * losses[0]


def test_durations_feed_a_graph():
    p = configs.graph_params(1)
    ns = measured.durations(p["hidden"], p["seq"], p["tp"], calls=3, replays=2)
    assert set(ns) == set(gpt1f1b.OPERATORS) and all(200 < v < 50_000_000 for v in ns.values())
    G = E.Graph(configs.graph(1, operator_ns=ns), 0)
    scen, n = E.scenarios_to_device(configs.scenario_batch(1), "cuda:0")
    assert int(G.compose(scen, n, 1)["step"][0]) > 0
    G.close()
