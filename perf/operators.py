"""Performance cases of the operators of a simulated training step: embedding, layer norm and cross
entropy, each with its gradient, through the package's public entry points.

A case is one operator at one size.  Keys (all plain values):
    op       "norm", "norm_grad", "embed", "embed_grad", "loss" (whole vocabulary, loss and gradient
             in one call) or "loss_shard" (one tensor-parallel rank's share of both)
    rows     tokens of the call
    cols     hidden size; for the losses, rows of the vocabulary held here
    type     element type of activations and weights
    residual norm: the residual stream is added first; norm_grad: its gradient is added to the result
    vocab    embed, embed_grad: rows of the vocabulary shard
    whole    embed, embed_grad, loss_shard: size of the whole vocabulary
    start    embed, embed_grad, loss_shard: first id of the shard
    ids      distribution of the token ids: "text" (the k-th id about 1/k as frequent as the first) or "even"
    index    "i32" or "i64": type of ids and targets
    main     norm_grad: weight gradients in 32 bits; embed_grad: a 32-bit gradient over two microbatches,
             the second added to the first

`run` has a plain form (elementary torch operations in 32 bits, rounded once) and, where `own` is true,
the calls of the package's operators.  Sizes: hidden 1024, 8192, 12288, sequences of 512 and 2048
and the vocabulary of 51200 over 1 to 8 tensor-parallel ranks are those of `workloads.configs`.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
VOCAB = 51200


def listed():
    return [
        # One new token of a small model: latency alone.
        dict(name="norm-1x1024", op="norm", rows=1, cols=1024, type="bf16", residual=False),
        # The tiny configuration's layer norm over one microbatch, in 32 bits.
        dict(name="norm-512x1024-f32", op="norm", rows=512, cols=1024, type="f32", residual=False),
        # A pre-norm block's entry at hidden size 8192: residual add and norm in one pass.
        dict(name="norm-res-2048x8192", op="norm", rows=2048, cols=8192, type="bf16", residual=True),
        # Backward of the tiny configuration's norm, main gradients in 32 bits.
        dict(name="normgrad-512x1024", op="norm_grad", rows=512, cols=1024, type="bf16", residual=False, main=True),
        # Odd sizes, half precision: rows that start at any element.
        dict(name="normgrad-1000x4099-f16", op="norm_grad", rows=1000, cols=4099, type="f16", residual=False, main=False),
        # The largest hidden size with the residual stream's gradient.
        dict(name="normgrad-res-2048x12288", op="norm_grad", rows=2048, cols=12288, type="bf16", residual=True, main=False),
        # A handful of new tokens looked up in the whole table.
        dict(name="embed-7x1024", op="embed", rows=7, cols=1024, type="bf16", vocab=VOCAB, whole=VOCAB, start=0,
             ids="text", index="i64"),
        # One of eight tensor-parallel ranks looks up eight microbatches; ids outside its shard give zeros.
        dict(name="embed-16384x8192-shard", op="embed", rows=16384, cols=8192, type="bf16", vocab=VOCAB // 8,
             whole=VOCAB, start=0, ids="text", index="i64"),
        # The tiny configuration's gradient over two microbatches into a 32-bit main gradient (TP 2).
        dict(name="embedgrad-512x1024-main", op="embed_grad", rows=512, cols=1024, type="bf16", vocab=VOCAB // 2,
             whole=VOCAB, start=0, ids="text", index="i64", main=True),
        # Eight microbatches at the largest hidden size, one of eight ranks: many tokens of few ids.
        dict(name="embedgrad-16384x12288", op="embed_grad", rows=16384, cols=12288, type="bf16", vocab=VOCAB // 8,
             whole=VOCAB, start=0, ids="text", index="i32", main=False),
        # The tiny configuration's loss on one of two vocabulary shards.
        dict(name="loss-512x25600-shard", op="loss_shard", rows=512, cols=VOCAB // 2, type="bf16", whole=VOCAB,
             start=VOCAB // 2, index="i64"),
        # A full microbatch over the whole vocabulary: loss and gradient of the logits.
        dict(name="loss-2048x51200", op="loss", rows=2048, cols=VOCAB, type="bf16", index="i64"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = {}


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16384 tokens, hidden sizes 33 to 16384, vocabularies of
    500 to 51200 rows in 1 to 8 shards, every type, no dearer than the operator's largest listed case."""
    if not _MOST:
        for c in listed():
            op = c["op"].replace("_shard", "")
            _MOST[op] = max(_MOST.get(op, 0), work(c)["bytes"])
    while True:
        op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "embed", "embed_grad", "embed_grad", "loss", "loss_shard"])
        c = dict(op=op, rows=_log(rng, 1, 4096), type=rng.choice(["bf16", "bf16", "f16", "f32"]))
        if op in ("norm", "norm_grad"):
            c.update(cols=_log(rng, 33, 16384), residual=rng.random() < 0.5)
            if rng.random() < 0.5:
                c["cols"] = -(-c["cols"] // 64) * 64
            if op == "norm_grad":
                c["main"] = rng.random() < 0.5
        else:
            shards = rng.choice([2, 4, 8] if op == "loss_shard" else [1, 2, 4, 8])
            c["index"] = rng.choice(["i32", "i64"])
            part = _log(rng, 500, VOCAB) // shards
            whole = part * shards
            start = part * rng.randrange(shards)
            if op == "loss":
                c["cols"] = whole
            elif op == "loss_shard":
                c.update(cols=part, whole=whole, start=start)
            else:
                c.update(rows=_log(rng, 1, 16384), cols=_log(rng, 33, 16384), vocab=part, whole=whole, start=start,
                         ids=rng.choice(["text", "text", "even"]))
                if rng.random() < 0.7:
                    c["cols"] = -(-c["cols"] // 64) * 64
                if op == "embed_grad":
                    c["main"] = rng.random() < 0.3
        if op in ("embed", "embed_grad") and _tokens(c)[0] < min(c["rows"], 8):
            continue  # a shard that no token falls into
        if c["cols"] == 3072 or work(c)["bytes"] > _MOST[op.replace("_shard", "")]:
            continue
        return c


def _ids(case, g, shape):
    whole = case["whole"]
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
    if case["ids"] == "text":
        ids = torch.exp(u * math.log(whole + 1)).long() - 1
    else:
        ids = (u * whole).long()
    return ids.clamp_(0, whole - 1).to(torch.int32 if case["index"] == "i32" else torch.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t = TYPES[case["type"]]
    r, c, op = case["rows"], case["cols"], case["op"]

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    s = dict(case=case, op=op)
    if op == "norm":
        # activations with an offset and a few large channels, as residual streams have
        channel = 1 + 4 * (torch.rand(c, generator=g, device="cuda") < 0.02)
        s["x"] = (torch.randn(r, c, generator=g, device="cuda") * channel + 1).to(t)
        s["residual"] = normal(r, c, std=0.5) if case["residual"] else None
        s["weight"], s["bias"] = normal(c, std=0.1, mean=1.0), normal(c, std=0.1)
    elif op == "norm_grad":
        x = torch.randn(r, c, generator=g, device="cuda") * 1.5 + 0.3
        s["x"] = x.to(t)
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
        s["weight"] = normal(c, std=0.1, mean=1.0)
        s["dy"] = normal(r, c, std=0.02, mean=0.002)
        s["dres"] = normal(r, c, std=0.02) if case["residual"] else None
    elif op == "embed":
        s["scale"] = math.sqrt(c)
        s["weight"] = normal(case["vocab"], c, std=0.02)
        s["ids"] = _ids(case, g, (r,))
    elif op == "embed_grad":
        s["scale"] = math.sqrt(c)
        n = 2 if case["main"] else 1
        s["ids"] = _ids(case, g, (n, r))
        s["dy"] = normal(n, r, c, std=0.01)
        if case["main"]:
            s["main"] = torch.empty(case["vocab"], c, device="cuda")
    else:
        whole = case.get("whole", c)
        s["logits"] = normal(r, c, std=2.5)
        targets = (torch.rand(r, generator=g, device="cuda", dtype=torch.float64) * whole).long().clamp_(0, whole - 1)
        # padding and prompts are not trained on
        targets = torch.where(torch.rand(r, generator=g, device="cuda") < 0.1, -100, targets)
        s["targets"] = targets.to(torch.int32 if case["index"] == "i32" else torch.int64)
        s["grad_loss"] = torch.full((r,), 1.0 / r, device="cuda")
        if op == "loss_shard":  # what the other ranks' shards add up to
            s["others"] = torch.randn(r, generator=g, device="cuda") * 0.1 + math.log(max(whole - c, 1)) + 2.5 ** 2 / 2
    return s


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2412_12487_amd as E

    case, op = s["case"], s["op"]
    if op == "norm":
        return E.layer_norm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual"])
    if op == "norm_grad":
        return E.layer_norm_grad(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], grad_residual=s["dres"],
                                 dtype=torch.float32 if case["main"] else None)
    if op == "embed":
        return E.embedding(s["ids"], s["weight"], s["scale"], vocab_start=case["start"])
    if op == "embed_grad":
        if not case["main"]:
            return E.embedding_grad(s["ids"][0], s["dy"][0], case["vocab"], s["scale"], vocab_start=case["start"])
        E.embedding_grad(s["ids"][0], s["dy"][0], case["vocab"], s["scale"], vocab_start=case["start"], out=s["main"])
        return E.embedding_grad(s["ids"][1], s["dy"][1], case["vocab"], s["scale"], vocab_start=case["start"],
                                out=s["main"], accumulate=True)
    if op == "loss":
        return E.cross_entropy(s["logits"], s["targets"], grad_loss=s["grad_loss"])
    part = E.cross_entropy(s["logits"], s["targets"], vocab_start=case["start"], vocab_size=case["whole"])
    lse = torch.logaddexp(part["lse"], s["others"])
    return {"target": part["target"], "lse": lse,
            "grad": E.cross_entropy_grad(s["logits"], s["targets"], lse, s["grad_loss"], vocab_start=case["start"],
                                         vocab_size=case["whole"])}


def _plain(s):
    case, op = s["case"], s["op"]
    if op == "norm":
        x, out = s["x"], {}
        if s["residual"] is not None:
            x = (x.float() + s["residual"].float()).to(x.dtype)
            out["sum"] = x
        x = x.float()
        out["mean"] = x.mean(1)
        x = x - out["mean"][:, None]
        out["rstd"] = torch.rsqrt((x * x).mean(1) + EPS)
        out["y"] = (x * out["rstd"][:, None] * s["weight"].float() + s["bias"].float()).to(s["x"].dtype)
        return out
    if op == "norm_grad":
        dy = s["dy"].float()
        n = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        to = torch.float32 if case["main"] else s["weight"].dtype
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * n).sum(0).to(to), "dbias": dy.sum(0).to(to)}
    if op == "embed":
        at = s["ids"].long() - case["start"]
        here = (at >= 0) & (at < case["vocab"])
        rows = s["weight"][at.clamp(0, case["vocab"] - 1)].float() * s["scale"]
        return (rows * here[:, None]).to(s["weight"].dtype)
    if op == "embed_grad":
        at = s["ids"].reshape(-1).long() - case["start"]
        here = (at >= 0) & (at < case["vocab"])
        dy = s["dy"].reshape(-1, case["cols"]).float() * (here[:, None] * s["scale"])
        dw = torch.zeros(case["vocab"], case["cols"], device="cuda")
        dw.index_add_(0, at.clamp(0, case["vocab"] - 1), dy)
        return dw if case["main"] else dw.to(s["dy"].dtype)
    x, start = s["logits"].float(), case.get("start", 0)
    targets = s["targets"].long()
    trained = (targets >= 0) & (targets < case.get("whole", case["cols"]))
    at = targets - start
    here = trained & (at >= 0) & (at < case["cols"])
    at = at.clamp(0, case["cols"] - 1)[:, None]
    target = torch.where(here, x.gather(1, at)[:, 0], 0.0)
    top = x.max(1).values
    lse = top + torch.log(torch.exp(x - top[:, None]).sum(1))
    if op == "loss_shard":
        top = torch.maximum(lse, s["others"])
        lse = top + torch.log(torch.exp(lse - top) + torch.exp(s["others"] - top))
    p = torch.exp(x - lse[:, None])
    p.scatter_add_(1, at, -here[:, None].float())
    grad = (p * (s["grad_loss"] * trained)[:, None]).to(s["logits"].dtype)
    if op == "loss_shard":
        return {"target": target, "lse": lse, "grad": grad}
    return {"loss": torch.where(trained, lse - target, 0.0), "lse": lse, "grad": grad}


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    w = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "norm":
        out, x = {}, w["x"]
        if case["residual"]:
            # the sum is an output of the activations' type, and what is normalised
            out["sum"] = x + w["residual"]
            x = out["sum"].to(s["x"].dtype).double()
        var, mean = torch.var_mean(x, 1, correction=0)
        out["mean"], out["rstd"] = mean, 1 / torch.sqrt(var + EPS)
        out["y"] = torch.addcmul(w["bias"], (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None], w["weight"])
        return out
    if op == "norm_grad":
        # through the Jacobian's two projections, rows as vectors
        n = torch.addcmul(-(w["mean"] * w["rstd"])[:, None], w["x"], w["rstd"][:, None])
        g = w["dy"] * w["weight"]
        along = (g * n).sum(1, keepdim=True) / case["cols"]
        dx = (g - g.sum(1, keepdim=True) / case["cols"] - along * n) * w["rstd"][:, None]
        if case["residual"]:
            dx += w["dres"]
        return {"dx": dx, "dweight": torch.sum(w["dy"] * n, 0), "dbias": torch.sum(w["dy"], 0)}
    if op == "embed":
        padded = torch.cat([w["weight"] * s["scale"], torch.zeros(1, case["cols"], device="cuda", dtype=torch.float64)])
        at = s["ids"].long() - case["start"]
        return padded[torch.where((at < 0) | (at >= case["vocab"]), case["vocab"], at)]
    if op == "embed_grad":
        at = s["ids"].reshape(-1).long() - case["start"]
        here = torch.nonzero((at >= 0) & (at < case["vocab"]))[:, 0]
        dw = torch.zeros(case["vocab"], case["cols"], device="cuda", dtype=torch.float64)
        return dw.index_put_((at[here],), w["dy"].reshape(-1, case["cols"])[here], accumulate=True) * s["scale"]
    x, targets = w["logits"], s["targets"].long()
    whole, start = case.get("whole", case["cols"]), case.get("start", 0)
    trained = ((targets >= 0) & (targets < whole)).double()
    hot = torch.arange(start, start + case["cols"], device="cuda") == targets[:, None]
    target = torch.where(hot, x, 0.0).sum(1)
    lse = torch.logsumexp(x, 1)
    if op == "loss_shard":
        lse = torch.logaddexp(lse, w["others"])
    grad = (torch.exp(x - lse[:, None]) - hot.double()) * (w["grad_loss"] * trained)[:, None]
    if op == "loss_shard":
        return {"target": target, "lse": lse, "grad": grad}
    return {"loss": (lse - target) * trained, "lse": lse, "grad": grad}


def _tokens(case):
    """(expected tokens with an id in the shard, expected distinct ids among them) of one batch."""
    k = np.arange(case["start"], case["start"] + case["vocab"], dtype=np.float64)
    p = np.log((k + 2) / (k + 1)) / math.log(case["whole"] + 1)
    if case["ids"] == "even":
        p = np.full(k.shape, 1 / case["whole"])
    seen = 1 - np.exp(case["rows"] * np.log1p(-np.minimum(p, 1 - 1e-12)))
    return case["rows"] * float(p.sum()), float(seen.sum())


def work(case):
    r, c, op, e = case["rows"], case["cols"], case["op"], SIZE[case["type"]]
    if op == "norm":
        return {"bytes": r * c * e * (4 if case["residual"] else 2) + 2 * c * e + 8 * r, "flops": 8 * r * c}
    if op == "norm_grad":
        return {"bytes": r * c * e * (4 if case["residual"] else 3) + c * e + 2 * c * (4 if case["main"] else e) + 8 * r,
                "flops": 14 * r * c}
    i = 8 if case["index"] == "i64" else 4
    if op == "embed":
        return {"bytes": r * i + (r + _tokens(case)[1]) * c * e, "flops": r * c}
    if op == "embed_grad":
        here, rows = _tokens(case)
        if case["main"]:  # every row written once, and the second batch's rows read and written again
            return {"bytes": 2 * (r * i + here * c * e) + (case["vocab"] + 2 * rows) * c * 4, "flops": 2 * here * c}
        return {"bytes": r * i + here * c * e + case["vocab"] * c * e, "flops": here * c}
    return {"bytes": 2 * r * c * e + r * (i + 12), "flops": 8 * r * c}
