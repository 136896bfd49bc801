"""Plain 64-bit forms of the training-step operators and the error bounds of 32-bit kernels for them.

Every bound follows from the arithmetic alone.  u = 2^-24 is the rounding of one 32-bit operation; a sum of n terms
taken by at least 64 lanes side by side has a chain of at most n / 64 + 32 additions, so its
error is at most u (n / 64 + 32) sum |terms|; a sum taken one after the other has a chain of n.  A result is
rounded once to its own type: relative error UNIT[type], or half a step of its smallest subnormal."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half the smallest step below the normal numbers (32-bit kernels may flush below 2^-126)
SMALL = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}


def chain(n):
    return n / 64 + 32


def close(got, want, err, what=""):
    """|got - want| within err (of the 32-bit arithmetic) and one rounding to got's type, element by element;
    NaN and infinities in the same places."""
    got64 = got.double()
    finite = torch.isfinite(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), f"{what}: NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got64[inf], want[inf]), f"{what}: infinities differ"
    bound = err + UNIT[got.dtype] * (want.abs() + err) + SMALL[got.dtype]
    off = (got64 - want).abs()
    bad = finite & ~(off <= bound)
    if bad.any():
        i = int(torch.nonzero(bad.reshape(-1))[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds; first at {i}: got "
                             f"{float(got64.reshape(-1)[i])!r}, want {float(want.reshape(-1)[i])!r}, "
                             f"bound {float(bound.expand_as(want).reshape(-1)[i])!r}")


def layer_norm(h, weight, bias, eps):
    """{name: (value, bound)} for rows h (already rounded where a residual was added)."""
    h, w = h.double(), weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    d = chain(h.shape[-1])
    mean = h.mean(-1, keepdim=True)
    c = h - mean
    var = (c * c).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    e_mean = U * (d + 2) * h.abs().mean(-1, keepdim=True)
    # squares about a mean that is off by e_mean: their mean grows by e_mean^2; then their own sum, 1 / sqrt
    e_rstd = rstd * (U * (d + 16) + e_mean ** 2 / (var + eps))
    y = c * rstd * w + b
    e_y = w.abs() * (rstd * e_mean + c.abs() * e_rstd) + 8 * U * ((c * rstd * w).abs() + b.abs())
    return {"mean": (mean[..., 0], e_mean[..., 0]), "rstd": (rstd[..., 0], e_rstd[..., 0]), "y": (y, e_y)}


def layer_norm_grad(dy, x, weight, mean, rstd, grad_residual=None, old=(None, None)):
    dy, x, w = (t.double().reshape(-1, t.shape[-1]) for t in (dy, x, weight))
    mean, rstd = mean.double().reshape(-1, 1), rstd.double().reshape(-1, 1)
    rows, cols = dy.shape
    d = chain(cols)
    n = (x - mean) * rstd
    g = dy * w
    s1, s2 = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dx = rstd * (g - s1 - n * s2)
    e_dx = U * rstd * (8 * g.abs() + (d + 8) * a1 + (d + 16) * n.abs() * a2)
    if grad_residual is not None:
        r = grad_residual.double().reshape(-1, cols)
        dx = dx + r
        e_dx = e_dx + U * (r.abs() + dx.abs())
    out = {"dx": (dx, e_dx)}
    for k, term, before in (("dweight", dy * n, old[0]), ("dbias", dy, old[1])):
        s, e = term.sum(0), U * (rows + 8) * term.abs().sum(0)
        if before is not None:
            s, e = s + before.double(), e + U * (s.abs() + before.double().abs())
        out[k] = (s, e)
    return out


def embedding_grad(ids, dy, vocab, scale, start, old=None):
    cols = dy.shape[-1]
    at = ids.reshape(-1).long() - start
    here = (at >= 0) & (at < vocab)
    rows, at = dy.double().reshape(-1, cols)[here], at[here]
    zero = torch.zeros(vocab, cols, dtype=torch.float64, device=dy.device)
    s = zero.index_add(0, at, rows) * scale
    count = torch.zeros(vocab, 1, dtype=torch.float64, device=dy.device)
    count.index_add_(0, at, torch.ones_like(at, dtype=torch.float64)[:, None])
    e = U * (count + 4) * zero.index_add(0, at, rows.abs()) * abs(scale)
    if old is not None:
        s = s + old.double()
        e = torch.where(count > 0, e + U * s.abs(), 0.0)
    return s, e


def cross_entropy(logits, targets, start, whole, lse=None, grad_loss=None):
    """lse: the whole vocabulary's, for a shard's gradient (float32, taken as it is)."""
    l = logits.double().reshape(-1, logits.shape[-1])
    rows, cols = l.shape
    t = targets.reshape(-1).long()
    trained = (t >= 0) & (t < whole)
    at = torch.where(trained, t - start, -1)
    hot = torch.arange(cols, device=l.device) == at[:, None]
    target = torch.where(hot, l, 0.0).sum(1)
    own = torch.logsumexp(l, 1)
    top = torch.where(torch.isfinite(l.max(1).values), l.max(1).values, 0.0)
    # every exponential: 4 units of its own and its argument's rounding, which weighs at most
    # x exp(-x) < 0.37 in the sum; then the sum, the logarithm and the addition
    e_own = U * (chain(cols) + 32) + 4 * U * (own.abs() + (own - top).abs())
    out = {"lse": (own, torch.nan_to_num(e_own, posinf=0.0)), "target": (target, torch.zeros_like(target))}
    gone = own == -math.inf
    loss = torch.where(trained, torch.where(gone, math.inf, own - target), 0.0)
    out["loss"] = (loss, torch.where(trained & torch.isfinite(loss), out["lse"][1] + U * loss.abs(), 0.0))
    if grad_loss is not None:
        e_l = out["lse"][1] if lse is None else torch.zeros(rows, dtype=torch.float64, device=l.device)
        lse = own if lse is None else lse.double().reshape(-1)
        g = grad_loss.double().reshape(-1, 1)
        x = l - lse[:, None]
        p = torch.exp(x)
        e_p = torch.where(p > 0, p * (e_l[:, None] + 8 * U + 4 * U * x.abs()), 0.0)
        live = (trained & (lse != -math.inf))[:, None]
        out["grad"] = (torch.where(live, (p - hot.double()) * g, 0.0),
                       torch.where(live, g.abs() * (e_p + 4 * U * (p + hot.double())), 0.0))
        out["grad"] = (out["grad"][0], torch.nan_to_num(out["grad"][1]))
    return out
