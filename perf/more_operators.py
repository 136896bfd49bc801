"""Performance cases of the losses at the end of a training step: cross entropy taken straight from the hidden states and
the output table, distillation from a teacher's top logits, and distillation taken straight from the hidden states; each
with its gradient, through the package's public entry points.

A case is one operator at one size.  Keys (all plain values):
    op       "linear_loss" (hidden states and table, one target a row), "distill" (logits, a teacher's top ids a row) or
             "linear_distill" (hidden states and table, a teacher's top ids a row)
    form     "loss" (the loss alone), "train" (whole vocabulary, loss and gradients in one call) or "shard" (one
             tensor-parallel rank's share: its statistics, their join with the other ranks', then its gradients)
    rows     tokens of the call
    hidden   hidden size (linear ones)
    vocab    rows of the vocabulary held here
    whole    size of the whole vocabulary
    start    first id held here
    type     element type of activations and weights; gradients have it too
    index    "i32" or "i64": type of targets and teacher ids
    top      ids that the teacher gives a row
    teacher  element type of the teacher's logits
    temp     temperature

Distillation: with q the softmax of the teacher's logits over its top ids and p the student's over the whole vocabulary, both
at temperature T, a row's loss is T^2 times the divergence of p from q, and its gradient with respect to the student's
logits T (p - q).  Ids outside the vocabulary are padding, a row of padding alone is not trained on.

`run` has a plain form (elementary torch operations in 32 bits, rounded once) and, where `own` is true, the calls of the
package's operators.  Hidden 1024 and 8192, sequences of 512 and 2048 and the vocabulary of 51200 over 1 to 8
tensor-parallel ranks are sizes of `workloads.configs`.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "i32": 4, "i64": 8}
VOCAB = 51200


def _linear(name, form, rows, hidden, type, index="i64", shards=1, rank=0, vocab=VOCAB):
    part = vocab // shards
    return dict(name=name, op="linear_loss", form=form, rows=rows, hidden=hidden, vocab=part, whole=part * shards,
                start=part * rank, type=type, index=index)


def _distill(name, op, form, rows, top, type, index="i64", hidden=0, shards=1, rank=0, vocab=VOCAB, teacher="f32", temp=2.0):
    part = vocab // shards
    c = dict(name=name, op=op, form=form, rows=rows, vocab=part, whole=part * shards, start=part * rank, type=type,
             index=index, top=top, teacher=teacher, temp=temp)
    if op == "linear_distill":
        c["hidden"] = hidden
    return c


def listed():
    return [
        # One token's log probability under a small model: the table is read once, latency counts.
        _linear("linloss-1x1024", "loss", 1, 1024, "bf16"),
        # Evaluation of a full sequence at hidden size 8192: loss alone.
        _linear("linloss-2048x8192", "loss", 2048, 8192, "bf16"),
        # The tiny configuration's head and loss of one microbatch with their gradients.
        _linear("linloss-train-512x1024", "train", 512, 1024, "bf16"),
        # A full microbatch at hidden size 8192 over the whole vocabulary.
        _linear("linloss-train-2048x8192", "train", 2048, 8192, "bf16", index="i32"),
        # One of eight tensor-parallel ranks, eight microbatches.
        _linear("linloss-shard-16384x8192", "shard", 16384, 8192, "bf16", shards=8, rank=2),
        # Odd sizes in 32 bits.
        _linear("linloss-train-500x1001-f32", "train", 500, 1001, "f32", vocab=4099),
        # A handful of tokens, the loss alone: latency.
        _distill("distill-7x51200-k8", "distill", "loss", 7, 8, "bf16"),
        # A full microbatch of logits with the teacher's top 64 of each token.
        _distill("distill-train-2048x51200-k64", "distill", "train", 2048, 64, "bf16", teacher="bf16"),
        # One of four ranks, odd sizes, half precision.
        _distill("distill-shard-1000x12801-k33-f16", "distill", "shard", 1000, 33, "f16", shards=4, rank=1, vocab=51204,
                 index="i32", temp=1.0),
        # The tiny configuration's head distilled in one call.
        _distill("lindistill-train-512x1024-k32", "linear_distill", "train", 512, 32, "bf16", hidden=1024),
        # A full microbatch at hidden size 8192 distilled in one call.
        _distill("lindistill-train-2048x8192-k64", "linear_distill", "train", 2048, 64, "bf16", hidden=8192, teacher="bf16"),
        # One of two ranks, half precision.
        _distill("lindistill-shard-1000x1024-k16-f16", "linear_distill", "shard", 1000, 16, "f16", hidden=1024, shards=2,
                 rank=1, index="i32", temp=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 1e15 * (4 if c["type"] == "f32" else 1)


_MOST = {}


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16384 tokens, hidden sizes 33 to 8192, vocabularies of 500 to 51200 rows
    in 1 to 8 shards, 1 to 128 teacher ids, every type, no dearer than the operator's largest listed case."""
    if not _MOST:
        for c in listed():
            _MOST[c["op"]] = max(_MOST.get(c["op"], 0), _cost(c))
    while True:
        op = rng.choice(["linear_loss", "linear_loss", "distill", "distill", "linear_distill"])
        form = rng.choice(["loss", "train", "train", "shard"])
        type = rng.choice(["bf16", "bf16", "f16", "f32"])
        shards = rng.choice([2, 4, 8]) if form == "shard" else 1
        vocab, rank, rows = _log(rng, 500, VOCAB), rng.randrange(shards), _log(rng, 1, 16384)
        index = rng.choice(["i32", "i64"])
        hidden = _log(rng, 33, 8192)
        if rng.random() < 0.7:
            hidden = -(-hidden // 64) * 64
        if rng.random() < 0.5:
            vocab = -(-vocab // 256) * 256
        if op == "linear_loss":
            c = _linear("", form, rows, hidden, type, index, shards, rank, vocab)
        else:
            c = _distill("", op, form, rows, _log(rng, 1, 128), type, index, hidden, shards, rank, vocab,
                         teacher=rng.choice(["f32", type]), temp=rng.choice([1.0, 2.0, 4.0]))
        del c["name"]
        if _cost(c) <= _MOST[op]:
            return c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t, op = TYPES[case["type"]], case["op"]
    r, v, whole, start = case["rows"], case["vocab"], case["whole"], case["start"]
    index = torch.int32 if case["index"] == "i32" else torch.int64

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float64)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = dict(case=case, op=op)
    if op == "linear_loss":
        ids = (uniform(r) * whole).long().clamp_(0, whole - 1)[:, None]
    else:
        k = case["top"]
        # distinct ids a row
        step = 1 + (uniform(r, 1) * (whole // k)).long().clamp_(0, whole // k - 1)
        first = (uniform(r, 1) * whole).long().clamp_(0, whole - 1)
        ids = (first + step * torch.arange(k, device="cuda")) % whole
    # how sure the student is of the first id, from not at all to altogether; of a sequence's first token never
    sure = (6 * uniform(r, 1)).float()
    sure[0] = 0
    at = ids[:, :1] - start
    here = (at >= 0) & (at < v)
    at = at.clamp(0, v - 1)
    if op == "distill":
        s["logits"] = normal(r, v, std=2.5).scatter_add_(1, at, 2.5 * sure * here).to(t)
    else:
        h = case["hidden"]
        s["weight"] = normal(v, h, std=2.5 / math.sqrt(h)).to(t)
        s["hidden"] = (normal(r, h) + sure / 2.5 * here * s["weight"][at[:, 0]].float()).to(t)
    if op == "linear_loss":
        # padding and prompts are not trained on
        skipped = uniform(r) < 0.1
        skipped[0] = False
        s["targets"] = torch.where(skipped, -100, ids[:, 0]).to(index)
    else:
        # a teacher's logits fall off over its top ids; some rows have fewer of them, and prompts none
        z = 12 + normal(r, k, std=2.0).sort(1, descending=True).values
        count = torch.where(uniform(r, 1) < 0.1, 0, torch.where(uniform(r, 1) < 0.2, 1 + (uniform(r, 1) * (k - 1)).long(), k))
        count[0] = k
        s["ids"] = torch.where(torch.arange(k, device="cuda") < count, ids, -1).to(index)
        s["teacher"] = z.to(TYPES[case["teacher"]])
    # half precision trains with its loss scaled up
    s["grad_loss"] = torch.full((r,), (1024.0 if case["type"] == "f16" else 1.0) / r, device="cuda")
    if case["form"] == "shard":  # what the other ranks' shards add up to
        temp = case.get("temp", 1.0)
        s["others"] = normal(r, std=0.1) + math.log(max(whole - v, 1)) + (2.5 / temp) ** 2 / 2
    return s


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2412_12487_amd as E

    case, op, form = s["case"], s["op"], s["case"]["form"]
    if op == "linear_loss":
        given, more = (s["hidden"], s["weight"], s["targets"]), {}
        loss, grad = E.linear_cross_entropy, E.linear_cross_entropy_grad
    else:
        given = (s["logits"],) if op == "distill" else (s["hidden"], s["weight"])
        given, more = given + (s["ids"], s["teacher"]), dict(temperature=case["temp"])
        loss, grad = (E.distillation, E.distillation_grad) if op == "distill" else (E.linear_distillation, E.linear_distillation_grad)
    if form == "loss":
        return loss(*given, **more)
    if form == "train":
        return loss(*given, grad_loss=s["grad_loss"], **more)
    more.update(vocab_start=case["start"], vocab_size=case["whole"])
    out = loss(*given, **more)
    out["lse"] = torch.logaddexp(out["lse"], s["others"])
    grads = grad(*given, out["lse"], s["grad_loss"], **more)
    return {**out, "grad": grads} if op == "distill" else {**out, **grads}


def _plain(s):
    case, op, form = s["case"], s["op"], s["case"]["form"]
    temp, v = case.get("temp", 1.0), case["vocab"]
    if op == "distill":
        x = s["logits"].float() / temp
    else:
        h, w = s["hidden"].float(), s["weight"].float()
        x = (h @ w.t()) / temp
    # a target is a teacher of one id
    ids = (s["targets"][:, None] if op == "linear_loss" else s["ids"]).long()
    z = torch.zeros(ids.shape, device="cuda") if op == "linear_loss" else s["teacher"].float() / temp
    known = (ids >= 0) & (ids < case["whole"])
    z = torch.where(known, z, -math.inf)
    top = z.max(1, keepdim=True).values
    trained = (top > -math.inf)[:, 0]
    q = torch.where(known, torch.exp(z - torch.where(trained[:, None], top, 0.0)), 0.0)
    total = q.sum(1, keepdim=True)
    q = q / torch.where(trained[:, None], total, 1.0)
    log_q = torch.where(q > 0, z - top - torch.log(total), 0.0)
    at = ids - case["start"]
    here = known & (at >= 0) & (at < v)
    at = at.clamp(0, v - 1)
    student = torch.where(here, x.gather(1, at), 0.0)
    m = x.max(1).values
    lse = m + torch.log(torch.exp(x - m[:, None]).sum(1))
    if form == "shard":
        out = {"target": (q * student).sum(1)}
        if op != "linear_loss":
            out["entropy"] = -(q * log_q).sum(1)
        m = torch.maximum(lse, s["others"])
        lse = m + torch.log(torch.exp(lse - m) + torch.exp(s["others"] - m))
    else:
        out = {"loss": temp * temp * (q * (log_q + (lse[:, None] - student))).sum(1)}
    out["lse"] = lse
    if form == "loss":
        return out
    p = torch.exp(x - lse[:, None])
    p.scatter_add_(1, at, -torch.where(here, q, 0.0))
    d = p * (s["grad_loss"] * trained * temp)[:, None]
    if op == "distill":
        out["grad"] = d.to(s["logits"].dtype)
    else:
        out["dhidden"] = (d @ w).to(s["hidden"].dtype)
        out["dweight"] = (d.t() @ h).to(s["weight"].dtype)
    return out


def exact(case, seed):
    s, op, form = prepare(case, seed), case["op"], case["form"]
    t, start, v, whole = case.get("temp", 1.0), case["start"], case["vocab"], case["whole"]
    if op == "distill":
        x = s["logits"].double()
    else:
        h, w = s["hidden"].double(), s["weight"].double()
        x = torch.mm(h, w.t())
    # the teacher's distribution over the whole vocabulary, and one column more for padding
    r = case["rows"]
    dense = torch.zeros(r, whole + 1, dtype=torch.float64, device="cuda")
    if op == "linear_loss":
        ids = torch.where((s["targets"] >= 0) & (s["targets"] < whole), s["targets"].long(), whole)[:, None]
        dense.scatter_(1, ids, 1.0)
        plogp = torch.zeros(r, dtype=torch.float64, device="cuda")
    else:
        ids = torch.where((s["ids"] >= 0) & (s["ids"] < whole), s["ids"].long(), whole)
        z = torch.where(ids < whole, s["teacher"].double() / t, -math.inf)
        q = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
        dense.scatter_add_(1, ids, q)
        plogp = torch.special.xlogy(q, q).sum(1)
    dense = dense[:, start:start + v]
    trained = (ids < whole).any(1).double()
    lse = torch.logsumexp(x / t, 1)
    cross = (dense * x).sum(1) / t
    if form == "shard":
        out = {"target": cross}
        if op != "linear_loss":
            out["entropy"] = -plogp
        lse = torch.logaddexp(lse, s["others"].double())
    else:
        out = {"loss": t ** 2 * trained * (plogp - cross + lse)}
    out["lse"] = lse
    if form == "loss":
        return out
    d = (torch.exp(x / t - lse[:, None]) - dense) * (t * trained * s["grad_loss"].double())[:, None]
    if op == "distill":
        out["grad"] = d
    else:
        out["dhidden"] = torch.mm(d, w)
        out["dweight"] = torch.mm(d.t(), h)
    return out


def work(case):
    r, v, e, op = case["rows"], case["vocab"], SIZE[case["type"]], case["op"]
    small = r * (8 if case["form"] == "loss" else 12)
    if op == "linear_loss":
        small += r * SIZE[case["index"]]
    else:
        small += r * case["top"] * (SIZE[case["index"]] + SIZE[case["teacher"]])
        if case["form"] == "shard":
            small += 4 * r
    grads = case["form"] != "loss"
    if op == "distill":
        return {"bytes": (2 if grads else 1) * r * v * e + small, "flops": (8 if grads else 4) * r * v}
    h = case["hidden"]
    return {"bytes": (2 if grads else 1) * (r + v) * h * e + small, "flops": (6 if grads else 2) * r * v * h}
