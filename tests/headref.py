"""Plain 64-bit forms of distillation and of the output head's losses, and the error bounds of the kernels for them.

U, UNIT, SMALL, chain and close are those of tests/opsref.py.  A product of n terms whose sums are taken in 32 bits in any order
is off by at most 2 U n sum |terms| (2 U: a matrix instruction may cut where another addition rounds).  An element of 32 bits is
the sum of three of 8 bits (bfloat16): of the nine products of two such elements six are summed, and the other three
are below 2^-24 + 2^-24 + 2^-32 of the whole, so that such a product has 6 n terms and 4 U sum |terms| more."""
from __future__ import annotations

import math

import torch

from tests.opsref import SMALL, U, UNIT, chain, close  # noqa: F401

# what the rounding of the logits' gradient may lose, and the smallest step it knows, relative to the largest |grad_loss|:
# half precision's shares are 2^14 times as large, 32 bits are three planes of 8
SHARE = {torch.float32: (2.0 ** -24, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -39), torch.bfloat16: (2.0 ** -8, 2.0 ** -126)}


def product(a, b, dtype, ea=None):
    """(a @ b in 64 bits, bound); ea: bounds of a's elements."""
    n = a.shape[1]
    size = a.abs() @ b.abs()
    e = size * (2 * U * 6 * n + 4 * U if dtype == torch.float32 else 2 * U * n)
    return a @ b, e if ea is None else e + ea @ b.abs()


def teacher(ids, z, whole, temp):
    """(mass of every entry, its bound, sum of q log q and its bound, rows trained on); entries outside [0, whole) have none."""
    ids, z = ids.reshape(-1, ids.shape[-1]).long(), z.double().reshape(-1, z.shape[-1]) / temp
    known = (ids >= 0) & (ids < whole)
    z = torch.where(known, z, -math.inf)
    trained = (z != -math.inf).any(1)
    q = torch.where(trained[:, None], torch.softmax(torch.where(trained[:, None], z, 0.0), 1), 0.0)
    size = torch.where(torch.isfinite(z), z.abs(), 0.0).max(1, keepdim=True).values
    rel = U * (chain(ids.shape[1]) + 32 + 8 * size)
    plogp = torch.special.xlogy(q, q)
    e_prior = (plogp.abs().sum(1) + 1) * (2 * rel[:, 0]) + rel[:, 0]
    return q, q * rel, plogp.sum(1), e_prior, trained


def loss(x, e_x, ids, q, e_q, prior, e_prior, trained, start, whole, temp, lse=None, grad_loss=None, kept=False):
    """{name: (value, bound)} for logits x (already divided by temp) that are off by e_x, entries `ids` of masses q.

    lse: the whole vocabulary's as given (32 bits, taken as it is), else the rows' own.  kept: exponentials are held as half
    precision (2^-11), 2^15 times as large (half a smallest step is 2^-40 of their part's largest, and that at most 1)."""
    rows, cols = x.shape
    own = torch.logsumexp(x, 1)
    top = torch.where(torch.isfinite(x), x, -math.inf).max(1).values
    top = torch.where(torch.isfinite(top), top, 0.0)
    worst = torch.where(torch.isfinite(x), e_x, 0.0).max(1).values
    # tiles' sums are taken relative to their own maximum and moved to the rows': some exponentials more a tile
    e_own = worst + U * (chain(cols) + 128) + 8 * U * (own.abs() + (own - top).abs())
    e_own = torch.nan_to_num(e_own, nan=0.0, posinf=0.0)
    at = ids - start
    here = (ids >= 0) & (ids < whole) & (at >= 0) & (at < cols) & (q != 0)
    at = at.clamp(0, cols - 1)
    hit = torch.where(here, x.gather(1, at), 0.0)
    e_hit = torch.where(here & torch.isfinite(hit), e_x.gather(1, at), 0.0)
    n = ids.shape[1]
    finite = torch.where(torch.isfinite(hit), hit, 0.0)
    cross = torch.where(here, q * hit, 0.0).sum(1)
    # sum of masses times logits, in any order, of logits or of their distance from the maximum
    far = torch.where(here & torch.isfinite(hit), (finite - top[:, None]).abs(), 0.0)

    def e_cross(size):
        return (q * e_hit + e_q * size + U * (n + 4) * q * size).sum(1)

    out = {"lse": (own, e_own), "target": (cross, e_cross(finite.abs())), "entropy": (-prior, e_prior)}
    value = temp * temp * (prior + own - cross)
    value = torch.where(trained, torch.where(own == -math.inf, math.inf, value), 0.0)
    e = temp * temp * (e_prior + e_own + e_cross(far) + 8 * U * (prior.abs() + (own - top).abs() + (q * far).sum(1)) + 2 * U * top.abs())
    out["loss"] = (value, torch.where(trained & torch.isfinite(value), e, 0.0))
    if grad_loss is not None:
        e_l = e_own if lse is None else torch.zeros_like(own)
        lse = own if lse is None else lse.double().reshape(-1)
        g = grad_loss.double().reshape(-1, 1) * temp
        far = x - lse[:, None]
        p = torch.exp(far)
        e_p = torch.where(p > 0, p * (e_x + e_l[:, None] + 16 * U + 4 * U * far.abs() + 2 * U * x.abs()), 0.0)
        if kept:
            e_p = e_p + p * 2.0 ** -11 + 2.0 ** -40
        mass = torch.zeros_like(x).scatter_add_(1, at, torch.where(here, q, 0.0))
        e_mass = torch.zeros_like(x).scatter_add_(1, at, torch.where(here, e_q + 4 * U * q, 0.0))
        live = (trained & (lse != -math.inf))[:, None]
        out["grad"] = (torch.where(live, (p - mass) * g, 0.0),
                       torch.nan_to_num(torch.where(live, g.abs() * (e_p + e_mass + 4 * U * (p + mass)), 0.0)))
    return out


def targets(t, whole):
    """One target a row as entries: (ids, q, e_q, prior, e_prior, trained)."""
    t = t.reshape(-1).long()
    trained = (t >= 0) & (t < whole)
    q = trained.double()[:, None]
    zero = torch.zeros_like(q[:, 0])
    return t[:, None], q, torch.zeros_like(q), zero, zero, trained


def entries(ids, z, whole, temp):
    return (ids.reshape(-1, ids.shape[-1]).long(), *teacher(ids, z, whole, temp))


def distillation(logits, ids, z, start, whole, temp, lse=None, grad_loss=None):
    x = logits.double().reshape(-1, logits.shape[-1]) / temp
    e_x = torch.where(torch.isfinite(x), 2 * U * x.abs(), 0.0)
    return loss(x, e_x, *entries(ids, z, whole, temp), start, whole, temp, lse, grad_loss)


def linear(hidden, weight, given, start, whole, temp=1.0, lse=None, grad_loss=None, old=None):
    """given: targets(...) or entries(...); old: what dweight is added to."""
    t = hidden.dtype
    h, w = hidden.double().reshape(-1, hidden.shape[-1]), weight.double()
    x, e_x = product(h, w.t(), t)
    x, e_x = x / temp, e_x / temp + 2 * U * (x / temp).abs()
    e_x = torch.nan_to_num(e_x, nan=0.0, posinf=0.0)
    out = loss(x, e_x, *given, start, whole, temp, lse, grad_loss, kept=t == torch.bfloat16 and lse is None)
    if grad_loss is None:
        return out
    d, e_d = out.pop("grad")
    # the share of each logit is rounded relative to the largest |grad_loss|
    most = grad_loss.abs().max().double() * temp
    rel, least = SHARE[t]
    e_d = e_d + (d.abs() + e_d) * (rel + 8 * U) + least * most
    out["dhidden"] = product(d, w, t, e_d)
    out["dweight"] = product(d.t(), h, t, e_d.t())
    out = {k: (v, e + 4 * U * v.abs() if k in ("dhidden", "dweight") else e) for k, (v, e) in out.items()}
    if old is not None:
        v, e = out["dweight"]
        out["dweight"] = v + old.double(), e + U * (v.abs() + old.double().abs())
    return out
