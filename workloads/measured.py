"""The operators of a pipeline stage outside its matrix products, run and timed on the GPU at hand.

    python -m workloads.measured 1        # config 1: durations of its operators, and its step time with them

`durations` times embedding, layer norm and cross entropy with their gradients at the sizes that one
tensor-parallel rank of a configuration has; `gpt1f1b.gpt_graph(..., operator_ns=...)` puts them in place of the
drawn durations of those ops, so that a simulated step rests on measured kernels there.
`training_step` runs the same operators together, as a GPT without the layers between its norms.
"""
from __future__ import annotations

import math
import sys

import torch

import paper_2412_12487_amd as E

from . import configs, gpt1f1b


def training_step(ids, targets, table, norms, *, scale=1.0, eps=1e-5, fused=False, teacher=None):
    """One forward and backward pass of: embedding, a chain of pre-norm blocks whose branch is the norm itself
    (h <- h + norm(h)), a last norm, logits over the same table, mean cross entropy over the trained tokens.

    ids, targets: [tokens]; table: [vocab, hidden]; norms: (weight, bias) of every block and of the last norm.
    Returns a dict: 'loss' (mean), 'table' (float32 gradient of the table, both uses added up; the product that gives the
    logits' use is rounded to the table's type first) and 'norms', a list of (weight gradient, bias gradient), float32.
    Nothing waits for the GPU.

    fused: the head and its loss are one operator, which returns no logits; the logits' use is then added up in 32 bits.
    teacher, with fused: (ids [tokens, top], logits, temperature) of a teacher whose mean distillation loss is added."""
    if teacher is not None and not fused:
        raise ValueError("a teacher needs the fused head")
    vocab = table.shape[0]
    h = E.embedding(ids, table, scale)
    saved, branch = [], None
    for weight, bias in norms:
        out = E.layer_norm(h, weight, bias, eps, residual=branch)
        h = out.get("sum", h)                 # the residual stream, which the next block reads again
        saved.append((h, out["mean"], out["rstd"]))
        branch = out["y"]
    trained = (targets >= 0) & (targets < vocab)
    grad_loss = trained.float() / trained.sum().clamp(min=1)
    past, grads = None, []
    if fused:
        out = E.linear_cross_entropy(branch, table, targets, grad_loss=grad_loss, dtype=torch.float32)
        loss, main, dy = (out["loss"] * grad_loss).sum(), out["dweight"], out["dhidden"]
        if teacher is not None:
            even = torch.full_like(grad_loss, 1 / len(grad_loss))
            out = E.linear_distillation(branch, table, teacher[0], teacher[1], temperature=teacher[2], grad_loss=even,
                                        out={"dweight": main}, accumulate=True)
            loss, dy = loss + (out["loss"] * even).sum(), dy + out["dhidden"]
    else:
        # the matrix products are the library's, and round their results once to the activations' type
        logits = branch @ table.t()
        out = E.cross_entropy(logits, targets, grad_loss=grad_loss, out={"grad": logits})
        loss = (out["loss"] * grad_loss).sum()
        main = (out["grad"].t() @ branch).float()
        dy = out["grad"] @ table
    for (weight, _), (h, mean, rstd) in zip(reversed(norms), reversed(saved)):
        g = E.layer_norm_grad(dy, h, weight, mean, rstd, grad_residual=past, dtype=torch.float32)
        grads.append((g["dweight"], g["dbias"]))
        dy = past = g["dx"]                   # of the stream, and of the branch added to it
    E.embedding_grad(ids, dy, vocab, scale, out=main, accumulate=True)
    return {"loss": loss, "table": main, "norms": grads[::-1]}


def operators(hidden, seq, tp=1, *, vocab=gpt1f1b.VOCAB, dtype=torch.bfloat16, seed=0, device=0):
    """{name of gpt1f1b.OPERATORS: call} of one microbatch of `seq` tokens on the first of `tp` tensor-parallel ranks,
    each on random data that it holds.  The frequent ids lie in that rank's shard of the vocabulary, so its lookup and its
    table's gradient take the longest of all ranks', which wait for it."""
    dev = torch.device("cuda", device)
    g = torch.Generator(device=dev).manual_seed(seed)
    here, whole = vocab // tp, vocab // tp * tp

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dtype)

    # the k-th id about 1 / k as frequent as the first, as in text
    u = torch.rand(seq, generator=g, device=dev, dtype=torch.float64)
    ids = (torch.exp(u * math.log(whole + 1)).long() - 1).clamp_(0, whole - 1)
    targets = torch.randint(0, whole, (seq,), generator=g, device=dev)
    table, x, dy, logits = normal(here, hidden, std=0.02), normal(seq, hidden), normal(seq, hidden), normal(seq, here, std=2.0)
    weight, bias = torch.ones(hidden, dtype=dtype, device=dev), torch.zeros(hidden, dtype=dtype, device=dev)
    stats = E.layer_norm(x, weight, bias)
    shard = dict(vocab_start=0, vocab_size=whole)
    lse = E.cross_entropy(logits, targets, **shard)["lse"] + math.log(tp)
    grad_loss = torch.full((seq,), 1.0 / seq, device=dev)
    main = torch.zeros(here, hidden, device=dev)
    return {
        "embed": lambda: E.embedding(ids, table),
        "norm": lambda: E.layer_norm(x, weight, bias),
        "loss": lambda: E.cross_entropy(logits, targets, **shard),
        "loss_grad": lambda: E.cross_entropy_grad(logits, targets, lse, grad_loss, **shard),
        "norm_grad": lambda: E.layer_norm_grad(dy, x, weight, stats["mean"], stats["rstd"], dtype=torch.float32),
        "embed_grad": lambda: E.embedding_grad(ids, dy, here, out=main, accumulate=True),
    }


def durations(hidden, seq, tp=1, *, calls=20, replays=5, **kw):
    """{operator: ns of one call} on the GPU: `calls` calls in a captured graph, replayed `replays` times and timed by
    events, so that the host's part, which a training step runs ahead of, is not in it.  The calls are all on the same
    tensors, which stay in the 256 MB cache as far as they fit: on others each time, hidden 12288 and 2048 tokens over 8 ranks,
    the lookup takes 17.5 us instead of 10.2, the norm 24.5 instead of 18.1, the loss's gradient 13.3 instead of 8.5."""
    ns = {}
    for name, call in operators(hidden, seq, tp, **kw).items():
        with torch.cuda.device(kw.get("device", 0)):
            call()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                for _ in range(calls):
                    call()
            graph.replay()
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            for _ in range(replays):
                graph.replay()
            end.record()
            end.synchronize()
            ns[name] = max(1, round(begin.elapsed_time(end) * 1e6 / (calls * replays)))
    return ns


def main(argv=None):
    argv = sys.argv[1:] if argv is None else argv
    config = int(argv[0]) if argv else 1
    p = configs.graph_params(config)
    ns = durations(p["hidden"], p["seq"], p["tp"])
    print(f"{configs.NAMES[config]}: one microbatch of {p['seq']} tokens, hidden {p['hidden']}, 1 of {p['tp']} ranks")
    for name in gpt1f1b.OPERATORS:
        print(f"  {name:10s} {ns[name] / 1e3:9.2f} us")
    scen, n = E.scenarios_to_device(configs.scenario_batch(config, n=1), "cuda:0")
    for what, graph in (("drawn", configs.graph(config)), ("measured", configs.graph(config, operator_ns=ns))):
        G = E.Graph(graph, 0)
        step = int(G.compose(scen, n, 1)["step"][0])
        G.close()
        print(f"  step with {what} durations of these operators: {step / 1e6:.3f} ms")
    return ns


if __name__ == "__main__":
    main()
