"""The training-step operators on the GPU against their plain 64-bit forms (tests/opsref.py).

Sizes from one element to rows wider than any variant holds in registers, odd sizes and strides, rows
that start at any element, masks that leave nothing, infinities and NaN, shards, accumulation, views,
offsets past 2^32 bytes, other streams and captured graphs."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2412_12487_amd as E
from tests import opsref as R

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, mean=0.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


def _odd(t, lead=3, pad=5):
    """t's values as a view whose rows start at odd elements of a wider buffer."""
    rows = t.reshape(-1, t.shape[-1])
    buf = torch.full((rows.shape[0], t.shape[-1] + lead + pad), 7.0, dtype=t.dtype, device=t.device)
    view = buf[:, lead:lead + t.shape[-1]]
    view.copy_(rows)
    return view


# ---------------------------------------------------------------- layer norm

# one element; below, at and over a load of 8; every width that some variant holds in registers, and past the last
WIDTHS = [1, 7, 8, 64, 65, 200, 512, 513, 1000, 1024, 1031, 2048, 2049, 4096, 4099, 8192, 8200, 12288, 16384, 16385,
          20000, 32768, 40001]
ROWS = [1, 2, 5, 67]


def _norm_case(rows, cols, dtype, wide, residual, seed, strided=False):
    g = _gen(seed)
    x = _normal(g, rows, cols, std=1.5, mean=0.7, dtype=dtype)
    r = _normal(g, rows, cols, std=0.5, dtype=dtype) if residual else None
    wt = F32 if wide else dtype
    w, b = _normal(g, cols, std=0.2, mean=1.0, dtype=wt), _normal(g, cols, std=0.3, dtype=wt)
    if strided:
        x, r = _odd(x), None if r is None else _odd(r, 1, 2)
    return x, r, w, b


def _check_norm(x, r, w, b, eps, **kw):
    out = E.layer_norm(x, w, b, eps, residual=r, **kw)
    h = x
    if r is not None:
        h = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(out["sum"], h)
    assert set(out) == ({"y", "mean", "rstd"} if r is None else {"y", "mean", "rstd", "sum"})
    for k, (v, e) in R.layer_norm(h, w, b, eps).items():
        R.close(out[k], v, e, k)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_widths(cols, dtype):
    for i, rows in enumerate(ROWS if cols < 5000 else [1, 3]):
        _check_norm(*_norm_case(rows, cols, dtype, i % 2 == 1, i % 2 == 0, 11 * cols + rows), 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [8, 515, 1024, 4099, 16384, 33000])
def test_layer_norm_views_and_shapes(cols, dtype):
    x, r, w, b = _norm_case(6, cols, dtype, False, True, cols, strided=True)
    _check_norm(x, r, w, b, 1e-5)
    _check_norm(x, None, w, None, 1e-3)
    once = _normal(_gen(3), 1, cols, dtype=dtype).expand(5, cols)      # one row repeated
    _check_norm(once, r[:5], w, b, 1e-5)
    x4 = _normal(_gen(4), 2, 3, 4, cols, dtype=dtype)
    out = E.layer_norm(x4, w, b)
    assert out["y"].shape == x4.shape and out["mean"].shape == (2, 3, 4)
    flat = E.layer_norm(x4.reshape(24, cols), w, b)
    assert torch.equal(out["y"].reshape(24, cols), flat["y"])
    one = E.layer_norm(x4[1, 2, 3], w, b)
    assert one["mean"].shape == () and torch.equal(one["y"], flat["y"][23])
    none = E.layer_norm(x4[:0], w, b)
    assert none["y"].shape == (0, 3, 4, cols)


def test_layer_norm_of_constant_rows_and_large_offsets():
    """Constant rows have variance 0 (rstd = 1 / sqrt(eps)); a large offset does not drown the variance."""
    w, b = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    for value in (0.0, 3.0, -1000.0):
        out = E.layer_norm(torch.full((3, 1000), value, device="cuda"), w, b, 1e-5)
        R.close(out["mean"], torch.full((3,), value, dtype=torch.float64, device="cuda"), abs(value) * 1000 * R.U)
    x = _normal(_gen(9), 40, 1000, std=0.01, mean=1000.0)
    _check_norm(x, None, w, b, 1e-8)
    y = E.layer_norm(torch.zeros(2, 1000, device="cuda"), w, b, 0.0)["y"]      # 0 * inf
    assert torch.isnan(y).all()


@pytest.mark.parametrize("cols", [100, 1024, 4100, 16384, 40000])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_layer_norm_bad_rows_stay_by_themselves(cols, bad):
    x, r, w, b = _norm_case(9, cols, BF16, False, True, cols)
    good = E.layer_norm(x, w, b, residual=r)
    x2 = x.clone()
    x2[4, cols - 1] = bad
    out = E.layer_norm(x2, w, b, residual=r)
    assert torch.isnan(out["y"][4].float()).all()
    keep = [0, 1, 2, 3, 5, 6, 7, 8]
    for k in out:
        assert torch.equal(out[k][keep], good[k][keep]), k


def test_layer_norm_outputs_in_place_of_inputs():
    x, r, w, b = _norm_case(33, 1500, BF16, False, True, 5)
    want = E.layer_norm(x, w, b, residual=r)
    x2, r2 = x.clone(), r.clone()
    out = E.layer_norm(x2, w, b, residual=r2, out={"sum": x2})
    assert out["sum"] is x2 and all(torch.equal(out[k], want[k]) for k in want)
    x2 = x.clone()
    out = E.layer_norm(x2, w, b, residual=r2, out={"sum": r2})
    assert out["sum"] is r2 and all(torch.equal(out[k], want[k]) for k in want)


def _grad_case(rows, cols, dtype, wide, residual, seed):
    g = _gen(seed)
    x, _, w, _ = _norm_case(rows, cols, dtype, wide, False, seed)
    s = E.layer_norm(x, w, None)
    dy = _normal(g, rows, cols, std=0.5, mean=0.05, dtype=dtype)
    dr = _normal(g, rows, cols, std=0.5, dtype=dtype) if residual else None
    return dy, x, w, s["mean"], s["rstd"], dr


def _check_norm_grad(dy, x, w, mean, rstd, dr, **kw):
    out = E.layer_norm_grad(dy, x, w, mean, rstd, grad_residual=dr, **kw)
    for k, (v, e) in R.layer_norm_grad(dy, x, w, mean, rstd, dr).items():
        if k in out:
            R.close(out[k].reshape(v.shape), v, e, k)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_grad_widths(cols, dtype):
    for i, rows in enumerate(ROWS if cols < 5000 else [1, 3]):
        _check_norm_grad(*_grad_case(rows, cols, dtype, i % 2 == 0, i % 2 == 1, 13 * cols + rows),
                         dtype=F32 if i >= 2 else None)


@pytest.mark.parametrize("rows,cols", [(300, 1024), (1111, 515), (2500, 64), (4097, 8), (700, 4099), (257, 12288),
                                       (520, 16391), (130, 20000)])
def test_layer_norm_grad_many_rows(rows, cols):
    _check_norm_grad(*_grad_case(rows, cols, BF16, False, True, rows), dtype=F32)
    _check_norm_grad(*_grad_case(rows, cols, F32, True, False, rows))


@pytest.mark.parametrize("cols", [9, 1030, 4096, 17000])
def test_layer_norm_grad_views_accumulation_and_no_bias(cols):
    dy, x, w, mean, rstd, dr = _grad_case(70, cols, F16, False, True, cols)
    want = _check_norm_grad(dy, x, w, mean, rstd, dr, dtype=F32)
    got = _check_norm_grad(_odd(dy), _odd(x, 1, 1), w, mean, rstd, _odd(dr, 2, 3), dtype=F32)
    assert all(torch.equal(got[k], want[k]) for k in want)
    _check_norm_grad(dy[:1].expand(70, cols), x, w, mean, rstd, None)
    assert "dbias" not in _check_norm_grad(dy, x, w, mean, rstd, dr, bias=False)
    g = _gen(1)
    for t in (F16, F32):
        old = _normal(g, cols, std=3.0, dtype=t), _normal(g, cols, std=3.0, dtype=t)
        out = E.layer_norm_grad(dy, x, w, mean, rstd, out={"dweight": old[0].clone(), "dbias": old[1].clone()},
                                accumulate=True)
        ref = R.layer_norm_grad(dy, x, w, mean, rstd, None, old)
        for k in ("dweight", "dbias"):
            R.close(out[k], *ref[k], k)
    inplace = dy.clone()
    out = E.layer_norm_grad(inplace, x, w, mean, rstd, grad_residual=dr, dtype=F32, out={"dx": inplace})
    assert out["dx"] is inplace and all(torch.equal(out[k], want[k]) for k in want)
    inplace = dr.clone()
    out = E.layer_norm_grad(dy, x, w, mean, rstd, grad_residual=inplace, dtype=F32, out={"dx": inplace})
    assert all(torch.equal(out[k], want[k]) for k in want)


def test_layer_norm_grad_of_no_rows():
    w = torch.ones(77, device="cuda")
    e = torch.empty(0, 77, device="cuda")
    s = torch.empty(0, device="cuda")
    out = E.layer_norm_grad(e, e, w, s, s)
    assert not out["dweight"].any() and not out["dbias"].any()
    keep = torch.full((77,), 2.5, device="cuda")
    out = E.layer_norm_grad(e, e, w, s, s, bias=False, out={"dweight": keep}, accumulate=True)
    assert (out["dweight"] == 2.5).all()


@pytest.mark.parametrize("cols", [300, 4096, 18000])
def test_layer_norm_grad_bad_rows_stay_by_themselves(cols):
    dy, x, w, mean, rstd, dr = _grad_case(9, cols, BF16, False, True, cols)
    good = E.layer_norm_grad(dy, x, w, mean, rstd, grad_residual=dr)
    dy2 = dy.clone()
    dy2[4, 3] = math.nan
    out = E.layer_norm_grad(dy2, x, w, mean, rstd, grad_residual=dr)
    keep = [0, 1, 2, 3, 5, 6, 7, 8]
    assert torch.equal(out["dx"][keep], good["dx"][keep]) and torch.isnan(out["dx"][4].float()).all()
    for k in ("dweight", "dbias"):      # the column's sum has it, the others do not
        nan = torch.isnan(out[k].float())
        assert nan[3] and int(nan.sum()) == 1
        assert torch.equal(out[k][~nan], good[k][~nan])


def _directional(f, x, v, h):
    return float((f(x + h * v) - f(x - h * v)) / (2 * h))


def _agrees(fd, grad, v):
    """A 32-bit gradient's elements are off by a few units times a chain of under 100: 1e-5 of the norms covers
    that, the differences' own error (h^2 and 2^-52 / h) is far below."""
    grad, v = grad.double(), v.double()
    assert abs(fd - float((grad * v).sum())) <= 1e-5 * float(grad.norm() * v.norm())


def test_layer_norm_grad_against_differences():
    g = _gen(21)
    x, w, b = _normal(g, 6, 50, mean=0.5), _normal(g, 50, mean=1.0, std=0.3), _normal(g, 50)
    dy = _normal(g, 6, 50)
    s = E.layer_norm(x, w, b, 1e-3)
    out = E.layer_norm_grad(dy, x, w, s["mean"], s["rstd"])

    def loss(x, w, b):
        return (R.layer_norm(x, w, b, 1e-3)["y"][0] * dy.double()).sum()

    x, w, b = x.double(), w.double(), b.double()
    for _ in range(3):
        v = _normal(g, 6, 50).double()
        _agrees(_directional(lambda t: loss(t, w, b), x, v, 1e-5), out["dx"], v)
        v = _normal(g, 50).double()
        _agrees(_directional(lambda t: loss(x, t, b), w, v, 1e-5), out["dweight"], v)
        _agrees(_directional(lambda t: loss(x, w, t), b, v, 1e-5), out["dbias"], v)


# ---------------------------------------------------------------- embedding

def _lookup(ids, weight, scale, start):
    at = ids.long() - start
    here = (at >= 0) & (at < weight.shape[0])
    if not weight.shape[0]:
        return torch.zeros(*ids.shape, weight.shape[1], dtype=weight.dtype, device=weight.device)
    rows = (weight[at.clamp(0, weight.shape[0] - 1)].float() * scale).to(weight.dtype)
    return torch.where(here[..., None], rows, torch.zeros((), dtype=weight.dtype, device=weight.device))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 8, 130, 512, 1024, 1031, 4096, 5000, 12288, 20001])
def test_embedding(cols, dtype):
    """One 32-bit product, rounded once: equal to the plain form."""
    g = _gen(cols)
    for tokens, vocab, start, index in ((1, 10, 0, torch.int64), (77, 50, 13, torch.int32), (600, 1000, 0, torch.int64)):
        w = _normal(g, vocab, cols, dtype=dtype)
        ids = torch.randint(0, 2 * vocab, (tokens,), generator=g, device="cuda").to(index)
        ids[-1] = start + vocab - 1
        for scale in (1.0, math.sqrt(cols)):
            assert torch.equal(E.embedding(ids, w, scale, vocab_start=start), _lookup(ids, w, scale, start))
    wide = _odd(w)
    assert torch.equal(E.embedding(ids, wide, 0.5), _lookup(ids, w, 0.5, 0))


def test_embedding_any_id_is_allowed():
    w = _normal(_gen(1), 5, 24)
    low, high = -2 ** 63, 2 ** 63 - 1
    ids = torch.tensor([0, 4, 5, -1, -100, low, high, 2 ** 32, 2 ** 32 + 1, 3], device="cuda")
    out = E.embedding(ids, w)
    want = torch.zeros(10, 24, device="cuda")
    want[0], want[1], want[9] = w[0], w[4], w[3]
    assert torch.equal(out, want)
    out = E.embedding(ids, w, vocab_start=2 ** 32)
    want.zero_()
    want[7], want[8] = w[0], w[1]
    assert torch.equal(out, want)
    assert torch.equal(E.embedding(ids.reshape(2, 5), w).reshape(10, 24), E.embedding(ids, w))
    assert E.embedding(ids[:0], w).shape == (0, 24)
    assert not E.embedding(ids, w[:0]).any()
    nan = w.clone()
    nan[1] = math.nan      # a row that no token names
    assert torch.equal(E.embedding(ids, nan), E.embedding(ids, w))


def _check_embedding_grad(ids, dy, vocab, scale, start, **kw):
    out = E.embedding_grad(ids, dy, vocab, scale, vocab_start=start, **kw)
    R.close(out, *R.embedding_grad(ids, dy, vocab, scale, start), "dweight")
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 64, 130, 512, 1031, 2048, 4100, 12288])
def test_embedding_grad_sizes(cols, dtype):
    g = _gen(cols)
    for tokens, vocab, start, index, wide in ((1, 3, 0, torch.int64, False), (50, 130, 7, torch.int32, True),
                                              (700, 64, 0, torch.int64, False), (1500, 900, 100, torch.int32, True)):
        ids = torch.randint(0, start + 2 * vocab, (tokens,), generator=g, device="cuda").to(index)
        ids[0] = start
        dy = _normal(g, tokens, cols, std=0.3, dtype=dtype)
        want = _check_embedding_grad(ids, dy, vocab, math.sqrt(cols), start, dtype=F32 if wide else None)
        got = E.embedding_grad(ids, _odd(dy), vocab, math.sqrt(cols), vocab_start=start, dtype=F32 if wide else None)
        assert torch.equal(want, got)


@pytest.mark.parametrize("tokens", [63, 64, 65, 127, 1000, 1024, 4096, 5001, 20000])
@pytest.mark.parametrize("kind", ["same", "two", "text", "distinct", "none"])
def test_embedding_grad_id_distributions(tokens, kind):
    """Every token with one id, runs that cross any split of the tokens, ids that all differ, none here."""
    g = _gen(tokens)
    vocab, cols, start = 6000, 72, 50
    if kind == "same":
        ids = torch.full((tokens,), start + 4097, device="cuda")
    elif kind == "two":
        ids = start + 63 + (torch.rand(tokens, generator=g, device="cuda") < 0.3).long()
    elif kind == "text":
        ids = torch.exp(torch.rand(tokens, generator=g, device="cuda") * math.log(vocab + 2 * start)).long()
    elif kind == "distinct":
        ids = torch.randperm(max(tokens, vocab) + 2 * start, generator=g, device="cuda")[:tokens]
    else:
        ids = torch.randint(0, start, (tokens,), generator=g, device="cuda")
    dy = _normal(g, tokens, cols, std=0.3, dtype=BF16)
    out = _check_embedding_grad(ids, dy, vocab, 1.5, start, dtype=F32)
    again = E.embedding_grad(ids, dy, vocab, 1.5, vocab_start=start, dtype=F32)
    assert torch.equal(out, again)      # no order of workgroups in the sums
    old = _normal(g, vocab, cols)
    acc = E.embedding_grad(ids, dy, vocab, 1.5, vocab_start=start, out=old.clone(), accumulate=True)
    R.close(acc, *R.embedding_grad(ids, dy, vocab, 1.5, start, old), "accumulated")
    old = old.to(BF16)
    acc = E.embedding_grad(ids, dy, vocab, 1.5, vocab_start=start, out=old.clone(), accumulate=True)
    R.close(acc, *R.embedding_grad(ids, dy, vocab, 1.5, start, old), "accumulated")


def test_embedding_grad_corner_ids_and_no_tokens():
    g = _gen(2)
    dy = _normal(g, 9, 40)
    ids = torch.tensor([-2 ** 63, 2 ** 63 - 1, -1, 0, 4, 5, 4, 2 ** 32 + 4, -100], device="cuda")
    _check_embedding_grad(ids, dy, 5, 2.0, 0)
    _check_embedding_grad(ids, dy, 5, 2.0, 2 ** 32)
    out = E.embedding_grad(ids[:0], dy[:0], 5)
    assert out.shape == (5, 40) and not out.any()
    keep = torch.full((5, 40), 2.5, device="cuda")
    assert (E.embedding_grad(ids[:0], dy[:0], 5, out=keep, accumulate=True) == 2.5).all()
    assert E.embedding_grad(ids, dy, 0).shape == (0, 40)
    row = dy[:1].expand(9, 40)      # a broadcast gradient
    _check_embedding_grad(ids, row, 5, 2.0, 0)
    bad = dy.clone()
    bad[0] = math.nan               # a token that is not here
    assert torch.equal(E.embedding_grad(ids, bad, 5), E.embedding_grad(ids, dy, 5))
    bad[3, 7] = math.nan
    out, good = E.embedding_grad(ids, bad, 5), E.embedding_grad(ids, dy, 5)
    nan = torch.isnan(out)
    assert int(nan.sum()) == 1 and nan[0, 7] and torch.equal(out[~nan], good[~nan])


def test_embedding_grad_against_differences():
    g = _gen(22)
    w, ids = _normal(g, 30, 20), torch.randint(0, 30, (40,), generator=g, device="cuda")
    dy = _normal(g, 40, 20)
    out = E.embedding_grad(ids, dy, 30, 3.0)
    v = _normal(g, 30, 20).double()
    _agrees(_directional(lambda t: (3.0 * t[ids] * dy.double()).sum(), w.double(), v, 1e-5), out, v)


# ---------------------------------------------------------------- cross entropy

LOSS_WIDTHS = [1, 2, 7, 8, 100, 512, 1000, 1024, 2047, 4096, 6400, 8193, 16384, 25600, 32769, 50257, 51200, 65536, 65537,
               131101]


def _loss_case(rows, cols, dtype, seed, whole=None, start=0, index=torch.int64, std=2.5):
    g = _gen(seed)
    whole = cols if whole is None else whole
    l = _normal(g, rows, cols, std=std, dtype=dtype)
    t = torch.randint(0, whole, (rows,), generator=g, device="cuda")
    if rows > 2:
        t[1] = -100
    return l, t.to(index), _normal(g, rows, std=0.5)


def _check_loss(l, t, gl, **kw):
    ref = R.cross_entropy(l, t, 0, l.shape[-1], grad_loss=gl)
    out = E.cross_entropy(l, t)
    assert set(out) == {"loss", "lse"}
    for k in out:
        R.close(out[k], *ref[k], k)
    full = E.cross_entropy(l, t, grad_loss=gl, **kw)
    assert set(full) == {"loss", "lse", "grad"}
    for k in full:
        R.close(full[k], *ref[k], k)
    ref = R.cross_entropy(l, t, 0, l.shape[-1], lse=out["lse"], grad_loss=gl)
    R.close(E.cross_entropy_grad(l, t, out["lse"], gl), *ref["grad"], "grad alone")
    return full


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", LOSS_WIDTHS)
def test_cross_entropy_widths(cols, dtype):
    for rows in ((1, 5, 70) if cols < 10000 else (1, 3)):
        index = torch.int32 if rows == 5 else torch.int64
        l, t, gl = _loss_case(rows, cols, dtype, cols + rows, index=index)
        full = _check_loss(l, t, gl)
        odd = E.cross_entropy(_odd(l), t, grad_loss=gl, out={"grad": _odd(l, 2, 1)})
        assert all(torch.equal(odd[k], full[k]) for k in full)
        same = l.clone()
        put = E.cross_entropy(same, t, grad_loss=gl, out={"grad": same})
        assert put["grad"] is same and all(torch.equal(put[k], full[k]) for k in full)
        same = l.clone()
        assert torch.equal(E.cross_entropy_grad(same, t, full["lse"], gl, out=same),
                           E.cross_entropy_grad(l, t, full["lse"], gl))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [9, 1000, 6400, 40000, 70000])
def test_cross_entropy_shards(cols, dtype):
    """Three ranks' shards join to the whole vocabulary's loss and gradient."""
    whole = 3 * cols
    l, t, gl = _loss_case(12, whole, dtype, cols)
    t[0], t[2], t[3], t[4] = 0, cols, whole - 1, whole      # edges; the last one is outside
    parts = []
    for k in range(3):
        piece = l[:, k * cols:(k + 1) * cols]
        p = E.cross_entropy(piece, t, vocab_start=k * cols, vocab_size=whole)
        assert set(p) == {"lse", "target"}
        ref = R.cross_entropy(piece, t, k * cols, whole)
        for name in p:
            R.close(p[name], *ref[name], name)
        parts.append(p)
    lse = torch.logsumexp(torch.stack([p["lse"] for p in parts]).double(), 0).float()
    loss = torch.where((t >= 0) & (t < whole), lse - sum(p["target"] for p in parts), 0.0)
    ref = R.cross_entropy(l, t, 0, whole)
    R.close(loss, ref["loss"][0], ref["lse"][1] + 8 * R.U * (lse.double().abs() + 10), "joined loss")
    for k in range(3):
        piece = l[:, k * cols:(k + 1) * cols]
        ref = R.cross_entropy(piece, t, k * cols, whole, lse=lse, grad_loss=gl)
        got = E.cross_entropy_grad(piece, t, lse, gl, vocab_start=k * cols, vocab_size=whole)
        R.close(got, *ref["grad"], "shard's gradient")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [70, 1024, 5000, 51200, 70001])
def test_cross_entropy_masks(cols, dtype):
    low = torch.finfo(dtype).min
    l, t, gl = _loss_case(10, cols, dtype, cols)
    t[:] = 3
    l[0] = -math.inf                       # nothing left
    l[1] = low                             # the lowest value everywhere: even
    l[2], l[2, 3] = -math.inf, 1.0         # the target alone is left
    l[3, 3] = -math.inf                    # the target is masked
    l[4, cols // 2:] = -math.inf
    l[5, cols // 2:] = low
    l[6] = low
    l[6, 3] = torch.finfo(dtype).max       # differences beyond the type's range
    l[7, :cols - 1] = -math.inf            # only the last column
    t[8] = -100
    l[8] = -math.inf                       # nothing left, and not trained on
    l[9] = 0.0
    full = _check_loss(l, t, gl)
    assert full["loss"][0] == math.inf and full["lse"][0] == -math.inf and not full["grad"][0].any()
    assert full["loss"][2] == 0 and full["loss"][3] == math.inf and full["loss"][8] == 0


@pytest.mark.parametrize("cols", [50, 4096, 51200, 70000])
def test_cross_entropy_bad_rows_stay_by_themselves(cols):
    l, t, gl = _loss_case(7, cols, BF16, cols)
    t[1] = 2
    good = E.cross_entropy(l, t, grad_loss=gl)
    bad = l.clone()
    bad[2, cols - 1], bad[4, 0] = math.nan, math.inf
    t2 = t.clone()
    t2[4] = -100                           # not trained on: its loss and gradient are zero all the same
    out = E.cross_entropy(bad, t2, grad_loss=gl)
    assert math.isnan(out["loss"][2]) and torch.isnan(out["grad"][2].float()).all()
    assert out["loss"][4] == 0 and not out["grad"][4].any()
    keep = [0, 1, 3, 5, 6]
    for k in out:
        assert torch.equal(out[k][keep], good[k][keep]), k
    t2[4] = 1
    out = E.cross_entropy(bad, t2, grad_loss=gl)
    assert math.isnan(out["loss"][4]) and torch.isnan(out["grad"][4].float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [70, 1024, 51200, 70001])
def test_cross_entropy_of_rows_masked_with_the_lowest_value(cols, dtype):
    """Every logit the same, however large: loss log(cols) and even probabilities, although the row's lse itself
    rounds the logarithm away.  A sum of cols equal terms 1 is off by a chain's roundings at most."""
    g = torch.tensor([1.0, 0.5, -2.0], device="cuda")
    l = torch.tensor([torch.finfo(dtype).min, -30000.0, 30000.0], device="cuda").to(dtype)[:, None].repeat(1, cols)
    t = torch.tensor([3, 0, cols - 1], device="cuda")
    out = E.cross_entropy(l, t, grad_loss=g)
    err = R.U * (R.chain(cols) + 32)
    want = torch.full((3,), math.log(cols), dtype=torch.float64, device="cuda")
    R.close(out["loss"], want, err + 2 * R.U * want, "loss")
    p = torch.full((3, cols), 1.0 / cols, dtype=torch.float64, device="cuda")
    hot = torch.nn.functional.one_hot(t, cols).double()
    R.close(out["grad"], (p - hot) * g.double()[:, None], (err * p + 4 * R.U * (p + hot)) * g.double().abs()[:, None], "grad")


def test_cross_entropy_shapes_and_targets_outside():
    l, t, gl = _loss_case(24, 300, F16, 1)
    t[5], t[6], t[7] = 300, 2 ** 62, -2 ** 63
    flat = _check_loss(l, t, gl)
    assert not flat["loss"][5:8].any() and not flat["grad"][5:8].any()
    cube = E.cross_entropy(l.reshape(2, 3, 4, 300), t.reshape(2, 3, 4), grad_loss=gl.reshape(2, 3, 4))
    assert cube["loss"].shape == (2, 3, 4) and torch.equal(cube["grad"].reshape(24, 300), flat["grad"])
    none = E.cross_entropy(l[:0], t[:0], grad_loss=gl[:0])
    assert none["loss"].shape == (0,) and none["grad"].shape == (0, 300)
    once = E.cross_entropy(l[:1].expand(24, 300), t, grad_loss=gl)
    ref = R.cross_entropy(l[:1].expand(24, 300), t, 0, 300, grad_loss=gl)
    for k in once:
        R.close(once[k], *ref[k], k)


def test_cross_entropy_grad_against_differences():
    g = _gen(23)
    l, t, gl = _loss_case(6, 60, F32, 23)
    out = E.cross_entropy(l, t, grad_loss=gl)

    def loss(x):
        return (R.cross_entropy(x, t, 0, 60)["loss"][0] * gl.double()).sum()

    for _ in range(3):
        v = _normal(g, 6, 60).double()
        _agrees(_directional(loss, l.double(), v, 1e-5), out["grad"], v)


# ---------------------------------------------------------------- all of them

def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes from the first: strides, tables, gradients and logits."""
    step = 1 << 28
    buf = torch.empty(9 * step, dtype=BF16, device="cuda")       # 4.8 GB
    x = torch.as_strided(buf, (9, 1000), (step, 1))
    x.copy_(_normal(_gen(1), 9, 1000))
    w, b = torch.ones(1000, dtype=BF16, device="cuda"), torch.zeros(1000, dtype=BF16, device="cuda")
    out = _check_norm(x, None, w, b, 1e-5)
    _check_norm_grad(x, x, w, out["mean"], out["rstd"], x)
    _check_loss(x, torch.arange(9, device="cuda"), torch.ones(9, device="cuda"))
    ids = torch.tensor([8, 0, 7, 3], device="cuda")
    assert torch.equal(E.embedding(ids, x, 2.0), _lookup(ids, x, 2.0, 0))
    _check_embedding_grad(torch.tensor([1, 1, 0, 2, 2, 2, 1, 0, 2], device="cuda"), x, 3, 1.0, 0)
    del buf, x
    vocab = 600_000                                              # a gradient of 4.9e9 bytes
    ids = torch.tensor([vocab - 1, 3, vocab - 1], device="cuda")
    dy = _normal(_gen(2), 3, 4096, dtype=BF16)
    out = E.embedding_grad(ids, dy, vocab)
    assert torch.equal(out[3], dy[1]) and torch.equal(out[-1], (dy[0].float() + dy[2].float()).to(BF16))
    assert not out[4:-1].any() and not out[:3].any()
    del out
    l = torch.empty(48_000, 51_200, dtype=BF16, device="cuda")   # 4.9e9 bytes
    l.zero_()
    l[-1, 5] = 9.0
    t = torch.full((48_000,), 5, device="cuda")
    out = E.cross_entropy(l, t, grad_loss=torch.ones(48_000, device="cuda"), out={"grad": l})
    ref = R.cross_entropy(torch.tensor([[0.0] * 5 + [9.0] + [0.0] * 51_194], device="cuda"), t[:1], 0, 51_200,
                          grad_loss=torch.ones(1, device="cuda"))
    R.close(out["loss"][-1:], *ref["loss"], "last row's loss")
    R.close(out["grad"][-1:], *ref["grad"], "last row's gradient")


def _everything(x, r, w, b, dy, ids, table, logits, targets, gl):
    n = E.layer_norm(x, w, b, residual=r)
    d = E.layer_norm_grad(dy, n["sum"], w, n["mean"], n["rstd"], grad_residual=r)
    e = E.embedding(ids, table, 2.0)
    de = E.embedding_grad(ids, dy, table.shape[0], 2.0)
    c = E.cross_entropy(logits, targets, grad_loss=gl)
    part = E.cross_entropy(logits, targets, vocab_start=0, vocab_size=logits.shape[1] + 50)
    cg = E.cross_entropy_grad(logits, targets, c["lse"], gl)
    return [n["y"], n["sum"], n["mean"], n["rstd"], d["dx"], d["dweight"], d["dbias"], e, de, c["loss"], c["lse"], c["grad"],
            part["lse"], part["target"], cg]


def _all_inputs(seed, rows=300, cols=1032, vocab=700):
    g = _gen(seed)
    x, r, w, b = _norm_case(rows, cols, BF16, False, True, seed)
    return [x, r, w, b, _normal(g, rows, cols, dtype=BF16), torch.randint(-5, vocab + 5, (rows,), generator=g, device="cuda"),
            _normal(g, vocab, cols, dtype=BF16), _normal(g, rows, 2000, std=2.0, dtype=BF16),
            torch.randint(-1, 2000, (rows,), generator=g, device="cuda"), _normal(g, rows)]


def test_the_same_bits_every_time_and_on_other_streams():
    args = _all_inputs(1)
    want = _everything(*args)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(_everything(*args), want))
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = [a.clone() for a in _all_inputs(2)]      # made on the side stream, behind other work
        for _ in range(5):
            big = big @ big * 1e-3
        for a, b in zip(late, args):
            a.copy_(b)
        got = _everything(*late)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_in_a_graph():
    """Replays follow the inputs' values, with eager work between them."""
    args = _all_inputs(3)
    _everything(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _everything(*args)
    for seed in (4, 5, 6):
        new = _all_inputs(seed)
        for a, b in zip(args, new):
            a.copy_(b)
        graph.replay()
        want = _everything(*new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_workspaces_may_be_shared_and_dirty():
    dy, x, w, mean, rstd, dr = _grad_case(500, 2050, BF16, False, True, 1)
    ids = torch.randint(0, 900, (500,), generator=_gen(1), device="cuda")
    want = E.layer_norm_grad(dy, x, w, mean, rstd), E.embedding_grad(ids, dy, 900)
    space = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        got = (E.layer_norm_grad(dy, x, w, mean, rstd, workspace=space),
               E.embedding_grad(ids, dy, 900, workspace=space))
        assert all(torch.equal(got[0][k], want[0][k]) for k in want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    x, r, w, b = _norm_case(4, 64, BF16, False, True, 1)
    s = E.layer_norm(x, w, b)
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    table, gl = _normal(_gen(1), 9, 64, dtype=BF16), torch.ones(4, device="cuda")
    f = torch.zeros(4, 64, device="cuda")
    ng = lambda **k: E.layer_norm_grad(*[k.pop(n, v) for n, v in (("dy", x), ("x", x), ("w", w), ("m", s["mean"]),
                                                                  ("k", s["rstd"]))], **k)
    bad = [
        (lambda: E.layer_norm(x.cpu(), w, b), "runs? on the GPU"),
        (lambda: E.layer_norm([1.0], w, b), "torch tensor"),
        (lambda: E.layer_norm(x.double(), w, b), "must be"),
        (lambda: E.layer_norm(x.t(), w[:4], b[:4]), "contiguous"),
        (lambda: E.layer_norm(x[:, ::2], w[:32], b[:32]), "contiguous"),
        (lambda: E.layer_norm(torch.zeros(3, 4, 64, device="cuda")[:, :2], w, b), "one run of rows"),
        (lambda: E.layer_norm(x, w[:63], b), "63 elements"),
        (lambda: E.layer_norm(x, w.half(), b), "weight must be"),
        (lambda: E.layer_norm(x, w, b.float()), "bias must be"),
        (lambda: E.layer_norm(x, w, b, -1.0), "eps"),
        (lambda: E.layer_norm(x, w, b, math.nan), "eps"),
        (lambda: E.layer_norm(x[:, :0], w[:0], b[:0]), "no elements"),
        (lambda: E.layer_norm(x, w, b, residual=r[:2]), "x's shape"),
        (lambda: E.layer_norm(x, w, b, residual=r.float()), "residual must be"),
        (lambda: E.layer_norm(x, w, b, out={"y": x}), "overlap"),
        (lambda: E.layer_norm(x, w, b, out={"sum": r}), "no entry 'sum'"),
        (lambda: E.layer_norm(x, w, b, out={"y": f}), "y must be"),
        (lambda: E.layer_norm(x, w, b, out={"mean": f[0]}), "shape"),
        (lambda: E.layer_norm(x[:3], w, b, residual=r[:3], out={"sum": x[1:]}), "overlap"),
        (lambda: ng(m=s["mean"][:3]), "3 elements"),
        (lambda: ng(m=s["mean"].half()), "mean must be"),
        (lambda: ng(x=f), "x must be"),
        (lambda: ng(dtype=torch.float16), "dtype must be"),
        (lambda: ng(accumulate=True), "accumulate"),
        (lambda: ng(out={"dx": x}), "dx overlaps x"),
        (lambda: ng(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), "workspace holds"),
        (lambda: ng(workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[1:]), "aligned"),
        (lambda: ng(grad_residual=f), "grad_residual must be"),
        (lambda: E.embedding(ids.float(), table), "ids must be"),
        (lambda: E.embedding(ids, table[0]), "matrix"),
        (lambda: E.embedding(ids, table, vocab_start=-1), "shard"),
        (lambda: E.embedding(ids, table, out=f), "out must be"),
        (lambda: E.embedding(torch.stack([ids, ids], 1)[:, 0], table), "contiguous"),
        (lambda: E.embedding(ids, table, out=table[:4]), "overlap"),
        (lambda: E.embedding_grad(ids, x[:3], 9), "shape of ids"),
        (lambda: E.embedding_grad(ids, x, -1), "vocab"),
        (lambda: E.embedding_grad(ids, x, 9, accumulate=True), "accumulate"),
        (lambda: E.embedding_grad(ids, x, 9, dtype=torch.float16), "dtype"),
        (lambda: E.embedding_grad(ids, x, 9, out=f), "out has shape"),
        (lambda: E.embedding_grad(ids, x, 4, out=x), "overlap"),
        (lambda: E.embedding_grad(ids, x, 9, workspace=torch.empty(4, dtype=torch.uint8, device="cuda")), "workspace holds"),
        (lambda: E.cross_entropy(x, ids[:3]), "leading shape"),
        (lambda: E.cross_entropy(x, ids.float()), "targets must be"),
        (lambda: E.cross_entropy(x, ids, vocab_start=3), "vocab_size"),
        (lambda: E.cross_entropy(x, ids, vocab_start=3, vocab_size=66), "passes the vocabulary"),
        (lambda: E.cross_entropy(x, ids, vocab_size=100, grad_loss=gl), "cross_entropy_grad"),
        (lambda: E.cross_entropy(x, ids, grad_loss=gl.half()), "grad_loss must be"),
        (lambda: E.cross_entropy(x, ids, out={"grad": x}), "no entry 'grad'"),
        (lambda: E.cross_entropy(x[:3], ids[:3], grad_loss=gl[:3], out={"grad": x[1:]}), "overlap"),
        (lambda: E.cross_entropy(x, ids, grad_loss=gl, out={"grad": x[:1].expand(4, 64)}), "overlap"),
        (lambda: E.cross_entropy_grad(x, ids, gl[:3], gl), "3 elements"),
        (lambda: E.cross_entropy_grad(x, ids, gl, gl, vocab_start=9), "vocab_size"),
    ]
    for call, msg in bad:
        with pytest.raises(E.EchoError, match=msg):
            call()
    torch.cuda.synchronize()
    assert torch.equal(E.layer_norm(x, w, b)["y"], s["y"])      # nothing was left behind
