"""The output head's losses and distillation at the calls that tests/test_gpu_head.py does not make, against 64 bits: every
statistic asked for together, logits far from zero, weights of rows not trained on, shards by tiles, few rows, repeated ids."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2412_12487_amd as E
from paper_2412_12487_amd import ops
from tests import headref as R

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
CODE = {F32: 0, F16: 1, BF16: 2}
FEW, TILES = (70, 64, 300), (1030, 64, 6000)      # rows of parts; tiles (423 middle ones)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _case(rows, cols, vocab, dtype, seed, whole=None, std=2.5):
    g = _gen(seed)
    h, w = _normal(g, rows, cols, dtype=dtype), _normal(g, vocab, cols, std=std / math.sqrt(cols), dtype=dtype)
    t = torch.randint(0, whole or vocab, (rows,), generator=g, device="cuda")
    t[1::7] = -100
    return h, w, t, torch.full((rows,), 1 / rows, device="cuda")


def _teacher(rows, top, whole, seed):
    g = _gen(seed)
    ids = torch.randint(0, whole, (rows, top), generator=g, device="cuda")
    ids[1::5, top // 2:] = -1
    ids[2::9] = -100
    return ids, _normal(g, rows, top, std=2.0) + 3


def _close(out, ref, keys=None):
    for k in keys or out:
        R.close(out[k].reshape(ref[k][0].shape), *ref[k], k)


# ---------------------------------------------------------------- every statistic in one call of the C library

def _stats(rows, names):
    return {k: torch.full((rows,), 7.0, device="cuda") if k in names else None for k in ("lse", "target", "entropy", "loss")}


def _pointers(s, *names):
    return [None if s[k] is None else s[k].data_ptr() for k in names]


def _distill_all(l, ids, z, temp, gl=None, names=("lse", "target", "entropy", "loss")):
    rows, cols = l.shape
    s, g = _stats(rows, names), None if gl is None else torch.empty_like(l)
    ops._check(ops._ops().echo_distillation(
        l.data_ptr(), cols, CODE[l.dtype], ids.data_ptr(), 1, z.data_ptr(), CODE[z.dtype], rows, cols, ids.shape[1], 0, cols, temp,
        *_pointers(s, "lse", "target", "entropy", "loss"), None if gl is None else gl.data_ptr(), None if gl is None else g.data_ptr(),
        cols, l.device.index, ops._stream(l.device.index)))
    return {k: v for k, v in {**s, "grad": g}.items() if v is not None}


def _linear_all(h, w, t, z=None, temp=1.0, gl=None, names=("lse", "target", "entropy", "loss")):
    (rows, cols), vocab, L = h.shape, w.shape[0], ops._ops()
    s = _stats(rows, names if z is not None else [k for k in names if k != "entropy"])
    dh, dw = (None, None) if gl is None else (torch.empty_like(h), torch.empty_like(w))
    mats = (h.data_ptr(), cols, w.data_ptr(), cols, CODE[h.dtype])
    top = 0 if z is None else t.shape[1]
    space = torch.empty(L.echo_linear_workspace(*mats, rows, cols, vocab, top, 1, int(gl is not None)), dtype=torch.uint8, device="cuda")
    tail = (*([None] * 3 if gl is None else (gl.data_ptr(), dh.data_ptr(), dw.data_ptr())), CODE[h.dtype], 0, space.data_ptr(), space.numel(),
            h.device.index, ops._stream(h.device.index))
    if z is None:
        rc = L.echo_linear_cross_entropy(*mats, t.data_ptr(), 1, rows, cols, vocab, 0, vocab, *_pointers(s, "lse", "target", "loss"), *tail)
    else:
        rc = L.echo_linear_distillation(*mats, t.data_ptr(), 1, z.data_ptr(), CODE[z.dtype], rows, cols, vocab, top, 0, vocab, temp,
                                        *_pointers(s, "lse", "target", "entropy", "loss"), *tail)
    ops._check(rc)
    return {k: v for k, v in {**s, "dhidden": dh, "dweight": dw}.items() if v is not None}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [5, 500, 5000, 40000, 70000])
def test_distillation_gives_every_statistic_together(cols, dtype):
    """Teams of one wavefront and of several, rows too wide for registers and of less than a piece.  Logits lie about 20, so that a
    sum of masses times logits and one of masses times distances from the maximum differ."""
    rows, temp = 9, 2.0
    g = _gen(cols)
    l, gl = (_normal(g, rows, cols, std=2.5) + 20).to(dtype), _normal(g, rows)
    ids, z = _teacher(rows, 4, cols, 3)
    ref = R.distillation(l, ids, z, 0, cols, temp, grad_loss=gl)
    _close(_distill_all(l, ids, z, temp), ref)
    full = _distill_all(l, ids, z, temp, gl)
    assert set(full) == {"lse", "target", "entropy", "loss", "grad"}
    _close(full, ref)
    for name in ("lse", "target", "entropy", "loss"):      # each by itself is the same number
        assert torch.equal(_distill_all(l, ids, z, temp, names=(name,))[name], full[name]), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
@pytest.mark.parametrize("teacher", [False, True])
def test_the_head_gives_every_statistic_together(rows, cols, vocab, dtype, teacher):
    h, w, t, gl = _case(rows, cols, vocab, dtype, 5)
    h[:, 0], w[:, 0] = 4, 5      # logits lie about 20
    if teacher:
        t, z = _teacher(rows, 6, vocab, 3)
        given, temp = R.entries(t, z, vocab, 2.0), 2.0
    else:
        z, given, temp = None, R.targets(t, vocab), 1.0
    ref = R.linear(h, w, given, 0, vocab, temp, grad_loss=gl)
    alone = _linear_all(h, w, t, z, temp)
    assert set(alone) == ({"lse", "target", "loss"} | ({"entropy"} if teacher else set()))
    _close(alone, ref)
    _close(_linear_all(h, w, t, z, temp, gl), ref)
    for name in alone:
        assert torch.equal(_linear_all(h, w, t, z, temp, names=(name,))[name], alone[name]), name


# ---------------------------------------------------------------- logits far from zero

def _far(rows, cols, vocab, dtype, e, seed):
    """Hidden states and table whose products are sign 2^e plus small multiples of that number's last place in 32 bits: every product and
    every sum is exact in them.  Their first column alone is large."""
    g = _gen(seed)
    a, b = 2.0 ** (e - e // 2), 2.0 ** (e // 2)
    unit = 2.0 ** (e - 23)
    h = torch.randint(-1, 2, (rows, cols), generator=g, device="cuda").float()
    w = torch.randint(-2, 3, (vocab, cols), generator=g, device="cuda").float() * unit
    h[:, 0], w[:, 0] = a, b
    h[::2, 0] = -a
    # numbers below 2^e have a last place of half the size, so that sums of both signs of the rest are exact
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    t[1::7] = -100
    h, w = h.to(dtype), w.to(dtype)
    x = h.double() @ w.double().t()
    assert torch.equal(x, x.float().double())
    return h, w, t, x


def _exp(d):
    """exp(d) and its bound, d the exact distance of each logit from what its exponential is relative to: the product of d and
    log2(e) / T is off by 3 roundings, the exponential by 2."""
    p = torch.exp(d)
    return p, p * R.U * (4 * d.abs() + 2)


def _softmax(x, dtype):
    """(largest logit, sum of exponentials relative to it and its bound, probabilities and theirs) of exact logits x in one call; tiles'
    sums move some exponentials more, and exponentials of bfloat16 may be kept as half precision of 2^15 times their size."""
    top = x.max(1, keepdim=True).values
    s, e_s = _exp(x - top)
    total = s.sum(1, keepdim=True)
    e_total = e_s.sum(1, keepdim=True) + R.U * (R.chain(x.shape[1]) + 128) * total
    e = s * 2.0 ** -11 + 2.0 ** -40 if dtype == BF16 else 0.0
    return top, total[:, 0], e_total[:, 0], s / total, (e_s + e + s * (e_total / total + 16 * R.U)) / total


def _check_far(got, h, w, x, q, gl, temp, p, e_p, dtype):
    """Gradients of the columns that are small, where nothing of the first one's size cancels."""
    trained = (q.sum(1) > 0)[:, None]
    g = gl.double()[:, None] * temp
    d = torch.where(trained, (p - q) * g, 0.0)
    rel, least = R.SHARE[dtype]
    e_d = torch.where(trained, g.abs() * (e_p + 4 * R.U * (p + q)), 0.0)
    e_d = e_d + (d.abs() + e_d) * (rel + 8 * R.U) + least * float(gl.abs().max()) * temp
    for name, (v, e) in (("dhidden", R.product(d, w.double()[:, 1:], dtype, e_d)),
                         ("dweight", R.product(d.t(), h.double()[:, 1:], dtype, e_d.t()))):
        assert torch.isfinite(got[name]).all(), name
        R.close(got[name][:, 1:].contiguous(), v, e + 4 * R.U * v.abs(), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
@pytest.mark.parametrize("e", [10, 20, 24, 27])
@pytest.mark.parametrize("what", ["loss", "one call", "given lse"])
def test_logits_far_from_zero(rows, cols, vocab, e, dtype, what):
    """Logits of 2^e and both signs, whose distances from each other 32 bits hold exactly: a row's loss and probabilities follow from
    those distances, whatever the logits' own size.  From a given lse, which is a number of 32 bits, probabilities follow from the exact
    distances from that number."""
    h, w, t, x = _far(rows, cols, vocab, dtype, e, e)
    gl = torch.full((rows,), 1 / rows, device="cuda")
    top, total, e_total, p, e_p = _softmax(x, dtype)
    trained = t >= 0
    q = torch.zeros_like(x).scatter_(1, t.clamp(min=0)[:, None], trained.double()[:, None])
    full = E.linear_cross_entropy(h, w, t, grad_loss=gl)
    more, e_more = torch.log(total), e_total / total + 4 * R.U * (torch.log(total) + 1)
    loss = torch.where(trained, more + (top - x.gather(1, t.clamp(min=0)[:, None]))[:, 0], 0.0)
    R.close(full["loss"], loss, torch.where(trained, e_more + 4 * R.U * loss, 0.0), "loss")
    R.close(full["lse"], top[:, 0] + more, e_more, "lse")
    if what == "one call":
        _check_far(full, h, w, x, q, gl, 1.0, p, e_p, dtype)
    elif what == "given lse":
        p, e_p = _exp(x - full["lse"].double()[:, None])
        alone = E.linear_cross_entropy_grad(h, w, t, full["lse"], gl)
        _check_far(alone, h, w, x, q, gl, 1.0, p, e_p + 16 * R.U * p, dtype)


@pytest.mark.parametrize("e", [20, 24])
def test_logits_far_from_zero_in_pieces(e):
    """More than 1 GiB of the logits' gradient, whose pieces' logits are made anew in the same call."""
    rows, cols, vocab = 8192, 64, 25000
    h, w, t, x = _far(rows, cols, vocab, F32, e, e)
    gl = torch.full((rows,), 1 / rows, device="cuda")
    p, e_p = _softmax(x, F32)[3:]
    q = torch.zeros_like(x).scatter_(1, t.clamp(min=0)[:, None], (t >= 0).double()[:, None])
    _check_far(E.linear_cross_entropy(h, w, t, grad_loss=gl), h, w, x, q, gl, 1.0, p, e_p, F32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
@pytest.mark.parametrize("power", [-7, -19])
@pytest.mark.parametrize("what", ["loss", "one call", "given lse"])
def test_small_temperatures(rows, cols, vocab, power, dtype, what):
    """Logits of about 16 over a temperature of 2^-7 or 2^-19, nearly the smallest that is taken: 2^11 and 2^23.  As in _far, products
    and sums are exact; the elements are normal numbers of every type."""
    g = _gen(power)
    temp = 2.0 ** power
    h = torch.randint(-1, 2, (rows, cols), generator=g, device="cuda").float() * 2.0 ** -6
    w = torch.randint(-2, 3, (vocab, cols), generator=g, device="cuda").float() * 2.0 ** (power + 7)
    h[:, 0], w[:, 0] = 4, 4
    h, w = h.to(dtype), w.to(dtype)
    x = h.double() @ w.double().t()
    assert torch.equal(x, x.float().double())
    x = x / temp
    ids = torch.randint(0, vocab // 4, (rows, 4), generator=g, device="cuda") * 4 + torch.arange(4, device="cuda")      # no id twice
    z = torch.randint(-2, 3, (rows, 4), generator=g, device="cuda").float() * temp
    gl = torch.full((rows,), 1 / rows, device="cuda")
    mass, e_mass, prior, e_prior, trained = R.teacher(ids, z, vocab, temp)
    assert trained.all()
    top, total, e_total, p, e_p = _softmax(x, dtype)
    q, e_q = torch.zeros_like(x).scatter_(1, ids, mass), torch.zeros_like(x).scatter_(1, ids, e_mass)
    full = E.linear_distillation(h, w, ids, z, temperature=temp, grad_loss=gl)
    far = top - x.gather(1, ids)
    more, cross = torch.log(total), (mass * far).sum(1)
    loss = temp * temp * (prior + more + cross)
    bound = temp * temp * (e_prior + e_total / total + (e_mass * far).sum(1) + 16 * R.U * (prior.abs() + cross + more + 1))
    R.close(full["loss"], loss, bound, "loss")
    if what == "one call":
        _check_far(full, h, w, x, q, gl, temp, p, e_p + e_q, dtype)
    elif what == "given lse":
        p, e_p = _exp(x - full["lse"].double()[:, None])
        alone = E.linear_distillation_grad(h, w, ids, z, full["lse"], gl, temperature=temp)
        _check_far(alone, h, w, x, q, gl, temp, p, e_p + 16 * R.U * p + e_q, dtype)


def _distinct(g, rows, top, cols):
    """Ids of which none comes twice in a row."""
    return torch.rand(rows, cols, generator=g, device="cuda").argsort(1)[:, :top].contiguous()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temp", [0.3, 1e-3, 1e-6])
@pytest.mark.parametrize("cols", [5, 500, 5000, 40000, 70000])
@pytest.mark.parametrize("what", ["one call", "given lse"])
def test_distillation_of_logits_far_from_zero(cols, temp, dtype, what):
    """Logits of 2^15 and both signs that differ by a few of their last places, over temperatures that are no powers of two: 10^5 to
    3 * 10^10.  From a given lse, which is a number of 32 bits, logits / T are such numbers too."""
    rows, top = 6, min(4, cols)
    g = _gen(cols)
    k = torch.randint(-8, 9, (rows, cols), generator=g, device="cuda").double()
    l = (2.0 ** 15 + k * 2.0 ** 15 * torch.finfo(dtype).eps).to(dtype)
    l[::2] *= -1
    ids = _distinct(g, rows, top, cols)
    z = torch.randint(-2, 3, (rows, top), generator=g, device="cuda").float()
    gl = _normal(g, rows)
    t32 = float(torch.tensor(temp))      # what the library takes
    mass, e_mass, prior, e_prior, _ = R.teacher(ids, z, cols, t32)
    full = E.distillation(l, ids, z, temperature=temp, grad_loss=gl)
    q, e_q = torch.zeros(rows, cols, dtype=torch.float64, device="cuda").scatter_(1, ids, mass), R.U * 4
    e_q = torch.zeros_like(q).scatter_(1, ids, e_mass + e_q * mass)
    if what == "one call":
        top, total, e_total, p, e_p = _softmax(l.double() / t32, F32)
        d = l.double() / t32 - top
        e_p = e_p + 2 * R.U * d.abs() * p      # 1 / T is rounded
        far = -d.gather(1, ids)
        e_total = e_total + (2 * R.U * d.abs() * torch.exp(d)).sum(1)
        more, cross = torch.log(total), (mass * far).sum(1)
        bound = t32 * t32 * (e_prior + e_total / total + (e_mass * far).sum(1) + 16 * R.U * (prior.abs() + cross + more + 1))
        R.close(full["loss"], t32 * t32 * (prior + more + cross), bound, "loss")
        grad = full["grad"]
    else:
        x = (l.float() * (1 / torch.tensor(temp))).double()      # rounded to 32 bits, as the lse is
        p, e_p = _exp(x - full["lse"].double()[:, None])
        grad = E.distillation_grad(l, ids, z, full["lse"], gl, temperature=temp)
    scale = (gl.double() * t32)[:, None]
    R.close(grad, (p - q) * scale, scale.abs() * (e_p + e_q + 8 * R.U * (p + q)), "grad")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
def test_a_given_lse_is_above_every_logit(rows, cols, vocab, dtype):
    """Logits of 5e6 at a temperature that is no power of two: as numbers of 32 bits none is above the lse, and no probability above 1."""
    temp = 3e-6
    h, w, _, x = _far(rows, cols, vocab, dtype, 4, 3)
    ids, z = torch.arange(rows, device="cuda")[:, None] % vocab, torch.zeros(rows, 1, device="cuda")
    gl = torch.full((rows,), 1 / rows, device="cuda")
    lse = E.linear_distillation(h, w, ids, z, temperature=temp)["lse"]
    x = (x.float() * (1 / torch.tensor(temp))).double()
    p, e_p = _exp(x - lse.double()[:, None])
    assert float(p.max()) <= 1
    q = torch.zeros_like(x).scatter_(1, ids, 1.0)
    got = E.linear_distillation_grad(h, w, ids, z, lse, gl, temperature=temp)
    _check_far(got, h, w, x, q, gl, float(torch.tensor(temp)), p, e_p + 16 * R.U * p, dtype)


@pytest.mark.parametrize("temp", [0.3, 1e-3, 1e-6])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20])
@pytest.mark.parametrize("where", ["logits", "rows of parts", "tiles"])
def test_teachers_logits_far_from_zero(where, size, temp):
    """A teacher whose logits differ by a few of their last places: its distribution follows from their distances.  The student's is even."""
    rows, cols, vocab = TILES if where == "tiles" else FEW
    g = _gen(3)
    ids = _distinct(g, rows, 5, vocab)
    z = size + torch.randint(0, 9, (rows, 5), generator=g, device="cuda") * (size * 2.0 ** -23)
    z[::2] *= -1
    ids[3, 2] = -1
    z[4, 1] = -math.inf
    gl = torch.full((rows,), 1 / rows, device="cuda")
    t32 = float(torch.tensor(temp))
    x = torch.where(ids >= 0, z.double(), -math.inf)
    d = (x - x.max(1, keepdim=True).values) / t32
    q = torch.softmax(d, 1)
    far = torch.where(q > 0, d.abs(), 0.0)
    e_q = q * R.U * (4 * far.max(1, keepdim=True).values + 64)
    plogp = torch.special.xlogy(q, q)
    e_prior = (e_q * (1 + torch.where(q > 0, torch.log(q).abs(), 0.0))).sum(1) + 16 * R.U * (plogp.abs().sum(1) + 1)
    dense = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda").scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, q, 0.0))
    e_dense = torch.zeros_like(dense).scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, e_q, 0.0))
    loss = t32 * t32 * (plogp.sum(1) + math.log(vocab))
    e_loss = t32 * t32 * (e_prior + 64 * R.U * math.log(vocab))
    if where == "logits":
        l = torch.zeros(rows, vocab, device="cuda")
        out = E.distillation(l, ids, z, temperature=temp, grad_loss=gl)
        scale = gl.double()[:, None] * t32
        R.close(out["grad"], (1 / vocab - dense) * scale, scale * (e_dense + 64 * R.U / vocab + 8 * R.U * dense), "grad")
        entropy = E.distillation(l, ids, z, temperature=temp, vocab_start=0, vocab_size=vocab)["entropy"]
    else:
        h, w = torch.zeros(rows, cols, device="cuda"), torch.randint(-2, 3, (vocab, cols), generator=g, device="cuda").float()
        out = E.linear_distillation(h, w, ids, z, temperature=temp, grad_loss=gl)
        zero = torch.full_like(dense, 1 / vocab)
        _check_far(out, h, w, None, dense, gl, t32, zero, e_dense + 64 * R.U * zero, F32)
        entropy = E.linear_distillation(h, w, ids, z, temperature=temp, vocab_start=0, vocab_size=vocab)["entropy"]
    R.close(entropy, -plogp.sum(1), e_prior, "entropy")
    R.close(out["loss"], loss, e_loss, "loss")


# ---------------------------------------------------------------- rows whose weight is not used

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
@pytest.mark.parametrize("teacher", [False, True])
@pytest.mark.parametrize("weight", [1e30, math.inf, -math.inf, math.nan])
def test_weights_of_rows_not_trained_on(rows, cols, vocab, dtype, teacher, weight):
    """Whatever grad_loss holds for a row that is not trained on, the others have their gradients."""
    h, w, t, gl = _case(rows, cols, vocab, dtype, 5)
    gl = gl * 1e4
    if teacher:
        ids, z = _teacher(rows, 6, vocab, 3)
        z[4] = -math.inf
        dead = R.teacher(ids, z, vocab, 1.0)[4].logical_not()
        call, grad, given = E.linear_distillation, E.linear_distillation_grad, (ids, z)
    else:
        dead = t < 0
        call, grad, given = E.linear_cross_entropy, E.linear_cross_entropy_grad, (t,)
    assert dead.any() and not dead.all()
    gl[dead] = 0
    want = call(h, w, *given, grad_loss=gl)
    bad = torch.where(dead, torch.full_like(gl, weight), gl)
    got = call(h, w, *given, grad_loss=bad)
    assert all(torch.equal(got[k], want[k]) for k in want)
    want, got = grad(h, w, *given, want["lse"], gl), grad(h, w, *given, want["lse"], bad)
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [FEW, TILES])
def test_an_infinite_weight_stays_in_its_row(rows, cols, vocab, dtype):
    h, w, t, gl = _case(rows, cols, vocab, dtype, 5)
    gl = gl * 1e7      # half precision holds no share of such a weight as it is
    want = E.linear_cross_entropy(h, w, t, grad_loss=gl)
    gl[3] = math.inf
    got = E.linear_cross_entropy(h, w, t, grad_loss=gl)
    others = torch.arange(rows, device="cuda") != 3
    assert t[3] >= 0 and torch.equal(got["dhidden"][others], want["dhidden"][others])
    assert not torch.isfinite(got["dhidden"][3]).all()


# ---------------------------------------------------------------- shards

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [(1030, 64, 6000), (2048, 128, 8900)])
def test_linear_shards_by_tiles(rows, cols, vocab, dtype):
    """Three ranks whose logits come in tiles: middle ones, and a launch of wide ones with middle ones behind it.  Each rank's statistics
    and gradients, and the sum of their shares of the hidden states' gradient against the whole vocabulary's."""
    ranks, temp = 3, 2.0
    whole = vocab * ranks
    h, w, t, g = _case(rows, cols, whole, dtype, vocab)
    ids, z = _teacher(rows, 12, whole, 3)
    for given, args, more, call, grad, names in (
            (R.targets(t, whole), (t,), {}, E.linear_cross_entropy, E.linear_cross_entropy_grad, {"lse", "target"}),
            (R.entries(ids, z, whole, temp), (ids, z), dict(temperature=temp), E.linear_distillation, E.linear_distillation_grad,
             {"lse", "target", "entropy"})):
        scale = temp if more else 1.0
        at = [dict(vocab_start=rank * vocab, vocab_size=whole, **more) for rank in range(ranks)]
        parts = [w[rank * vocab:(rank + 1) * vocab] for rank in range(ranks)]
        stats, bounds = [], []
        for rank in range(ranks):
            out, ref = call(h, parts[rank], *args, **at[rank]), R.linear(h, parts[rank], given, rank * vocab, whole, scale)
            assert set(out) == names
            _close(out, ref)
            stats.append(out)
            bounds.append({k: ref[k][1] + R.U * (ref[k][0].abs() + ref[k][1]) for k in names})
        lse = torch.logsumexp(torch.stack([s["lse"] for s in stats]), 0)
        dh = bound = 0
        for rank in range(ranks):
            out = grad(h, parts[rank], *args, lse, g, **at[rank])
            ref = R.linear(h, parts[rank], given, rank * vocab, whole, scale, lse=lse, grad_loss=g)
            _close(out, ref)
            dh, bound = dh + out["dhidden"].double(), bound + ref["dhidden"][1] + R.UNIT[dtype] * (ref["dhidden"][0].abs() + ref["dhidden"][1])
        value = R.linear(h, w, given, 0, whole, scale, lse=lse, grad_loss=g)["dhidden"][0]
        assert ((dh - value).abs() <= bound + R.SMALL[dtype] * ranks).all()
        # the joined loss is the whole vocabulary's; the join itself is a few roundings of its result
        joined = lse.double() - sum(s["target"].double() for s in stats) - (stats[0]["entropy"].double() if more else 0)
        e = torch.stack([b["lse"] for b in bounds]).max(0).values + 16 * R.U * (lse.double().abs() + 1)
        e = e + sum(b["target"] for b in bounds) + (bounds[0]["entropy"] if more else 0)
        value, trained = R.linear(h, w, given, 0, whole, scale)["loss"][0], given[5]
        assert trained.any() and ((scale * scale * joined - value).abs() <= scale * scale * e)[trained].all()


# ---------------------------------------------------------------- few rows, repeated ids

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [1, 2, 64])
def test_shares_of_few_rows_have_two_planes(rows, dtype):
    """Of up to 64 rows the logits' gradient is held in twice the bits: with the table's gradient in 32 bits nothing is off by a
    rounding to the type.  Products of small whole numbers, so that the logits are exact; half precision's smallest step is 2^-39 of the
    largest weight."""
    cols, vocab = 64, 300
    g = _gen(rows)
    h = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").to(dtype)
    w = (torch.randint(-2, 3, (vocab, cols), generator=g, device="cuda") / 16).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    gl = torch.linspace(1, 2, rows, device="cuda")
    rel, least = R.SHARE[dtype]
    out = E.linear_cross_entropy(h, w, t, grad_loss=gl, dtype=F32)
    got = {"one call": out["dweight"], "from lse": E.linear_cross_entropy_grad(h, w, t, out["lse"], gl, dtype=F32)["dweight"]}
    x = h.double() @ w.double().t()
    for name, lse in (("one call", None), ("from lse", out["lse"])):
        d, e_d = R.loss(x, torch.zeros_like(x), *R.targets(t, vocab), 0, vocab, 1.0, lse, gl)["grad"]
        e_d = e_d + (d.abs() + e_d) * (rel * rel + 8 * R.U) + least * float(gl.max())
        v, e = R.product(d.t(), h.double(), dtype, e_d.t())
        e = e + e * 0.01 + 4 * R.U * v.abs()      # the second plane's own sum is 2^-8 of the first's at most
        R.close(got[name], v, e, name)
        # one plane alone would be off by more
        one = (d / gl.max().double()).float().to(dtype).double() * gl.max().double()
        assert ((one.t() @ h.double() - v).abs() > 2 * (e + R.U * v.abs())).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_repeated_ids_in_tiles(dtype):
    """1024 entries a row whose ids come several times, where a tile's entries are in cells."""
    rows, cols, vocab = TILES
    h, w, _, g = _case(rows, cols, vocab, dtype, 2)
    gen = _gen(9)
    ids = torch.randint(0, vocab, (rows, 1024), generator=gen, device="cuda")
    z = _normal(gen, rows, 1024)
    ids[0] = 7
    ids[1::4, 1::2] = ids[1::4, 0::2]
    ids[2::4, 512:] = ids[2::4, :1]
    z[2::4, 0] = -math.inf
    _close(E.linear_distillation(h, w, ids, z, grad_loss=g), R.linear(h, w, R.entries(ids, z, vocab, 1.0), 0, vocab, grad_loss=g))


def test_an_id_named_twice():
    """Masses of an id add up in the gradient, in the cross term and in a shard's target; sum of q log q is over the entries, each with
    its own mass.  A student certain of an id that is named twice with equal logits has a loss of -T^2 log 2, and one that is merged
    into a single entry 0; their gradients are the same."""
    temp, ln2 = 2.0, math.log(2.0)
    for cols in (5, 700, 40000, 70000):
        l = torch.full((2, cols), -math.inf, device="cuda")
        l[:, 3] = 1.0
        ids = torch.tensor([[3, 3], [3, -1]], device="cuda")
        z = torch.tensor([[0.5, 0.5], [0.5 + temp * ln2, 0.0]], device="cuda")
        gl = torch.ones(2, device="cuda")
        out = E.distillation(l, ids, z, temperature=temp, grad_loss=gl)
        assert abs(float(out["loss"][0]) + temp * temp * ln2) < 1e-5 and abs(float(out["loss"][1])) < 1e-5
        assert float(out["grad"].abs().max()) < 1e-6
        shard = E.distillation(l, ids, z, temperature=temp, vocab_start=0, vocab_size=cols + 7)
        assert abs(float(shard["entropy"][0]) - ln2) < 1e-6 and float(shard["entropy"][1]) == 0
        assert torch.allclose(shard["target"], torch.full((2,), 0.5, device="cuda"), atol=1e-6)
        away = E.distillation(l, ids, z, temperature=temp, vocab_start=9, vocab_size=cols + 9)      # the id is another rank's
        assert torch.equal(away["entropy"], shard["entropy"]) and not away["target"].any()
    for rows, cols, vocab in (FEW, TILES):
        h, w, _, gl = _case(rows, cols, vocab, F32, 4)
        ids, z = _teacher(rows, 4, vocab // 4, 3)
        ids = torch.where(ids < 0, ids, ids * 4 + torch.arange(4, device="cuda"))      # no id twice
        split, halves = torch.cat([ids, ids], 1), torch.cat([z, z], 1)
        one = E.linear_distillation(h, w, ids, z, temperature=temp, grad_loss=gl)
        two = E.linear_distillation(h, w, split, halves, temperature=temp, grad_loss=gl)
        trained = (ids >= 0).any(1)
        assert torch.allclose(two["loss"], torch.where(trained, one["loss"] - temp * temp * ln2, 0.0), atol=1e-4)
        for k in ("dhidden", "dweight"):
            assert float((two[k] - one[k]).abs().max()) <= 1e-5 * float(one[k].abs().max()), k
