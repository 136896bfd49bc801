"""The output head's losses and distillation on the GPU against their plain 64-bit forms (tests/headref.py).

Sizes from one element to several tiles of every shape, odd sizes and strides, rows that are not trained on, teachers without
an id, ids that come twice, infinities and NaN, shards, pieces of the vocabulary, accumulation, streams and graphs."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2412_12487_amd as E
from tests import headref as R

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _odd(t, lead=3, pad=5):
    """t's values as a view whose rows start at odd elements of a wider buffer."""
    buf = torch.full((t.shape[0], t.shape[1] + lead + pad), math.nan, dtype=t.dtype, device=t.device)
    view = buf[:, lead:lead + t.shape[1]]
    view.copy_(t)
    return view


def _case(rows, cols, vocab, dtype, seed, whole=None, std=2.5, index=torch.int64):
    g = _gen(seed)
    h, w = _normal(g, rows, cols, dtype=dtype), _normal(g, vocab, cols, std=std / math.sqrt(cols), dtype=dtype)
    t = torch.randint(0, whole or vocab, (rows,), generator=g, device="cuda")
    t[1::7] = -100
    return h, w, t.to(index), torch.full((rows,), 1 / rows, device="cuda")


def _teacher(rows, top, whole, seed, dtype=F32, index=torch.int64):
    """Entries of which some ids come twice, some are padding, and some rows have none."""
    g = _gen(seed)
    ids = torch.randint(0, whole, (rows, top), generator=g, device="cuda")
    if top > 2:
        ids[::3, 2] = ids[::3, 0]
        ids[1::5, top // 2:] = -1
    ids[2::9] = -100
    return ids.to(index), _normal(g, rows, top, std=2.0, dtype=dtype) + 3


def _close(out, ref, keys=None):
    for k in keys or out:
        R.close(out[k].reshape(ref[k][0].shape), *ref[k], k)


# sizes: one element; below, at and over a step of the sum, a tile of every shape, a whole wave of workgroups
SIZES = [(1, 1, 1), (1, 64, 1), (2, 7, 3), (5, 64, 255), (64, 64, 256), (65, 128, 257), (129, 100, 1000), (300, 192, 700),
         (257, 320, 513), (520, 65, 3000), (33, 1031, 2050), (40, 128, 20000), (3, 2112, 17000), (700, 72, 12000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", SIZES)
def test_linear_cross_entropy_sizes(rows, cols, vocab, dtype):
    h, w, t, g = _case(rows, cols, vocab, dtype, rows + cols + vocab, index=torch.int32 if rows % 2 else torch.int64)
    ref = R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g)
    out = E.linear_cross_entropy(h, w, t)
    assert set(out) == {"loss", "lse"}
    _close(out, ref)
    full = E.linear_cross_entropy(h, w, t, grad_loss=g)
    assert set(full) == {"loss", "lse", "dhidden", "dweight"}
    assert full["dhidden"].dtype == full["dweight"].dtype == dtype
    _close(full, ref)
    alone = E.linear_cross_entropy_grad(h, w, t, out["lse"], g)
    ref = R.linear(h, w, R.targets(t, vocab), 0, vocab, lse=out["lse"], grad_loss=g)
    _close(alone, ref)
    odd = E.linear_cross_entropy(_odd(h), _odd(w, 1, 2), t, grad_loss=g)
    assert all(torch.equal(odd[k], full[k]) for k in full)      # laid out in order first
    again = E.linear_cross_entropy(h, w, t, grad_loss=g)
    assert all(torch.equal(again[k], full[k]) for k in full)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab,top", [(1, 1, 1, 1), (3, 64, 5, 2), (64, 64, 256, 7), (129, 100, 1000, 64), (300, 192, 700, 33),
                                                 (70, 128, 3001, 1024), (40, 128, 20000, 130), (700, 72, 12000, 5)])
def test_linear_distillation_sizes(rows, cols, vocab, top, dtype):
    h, w, _, g = _case(rows, cols, vocab, dtype, rows + cols + vocab)
    index, temp = (torch.int32, 2.0) if rows % 2 else (torch.int64, 1.7)
    ids, z = _teacher(rows, top, vocab, top, dtype if rows % 3 else F32, index)
    given = R.entries(ids, z, vocab, temp)
    ref = R.linear(h, w, given, 0, vocab, temp, grad_loss=g)
    out = E.linear_distillation(h, w, ids, z, temperature=temp)
    assert set(out) == {"loss", "lse"}
    _close(out, ref)
    full = E.linear_distillation(h, w, ids, z, temperature=temp, grad_loss=g)
    assert set(full) == {"loss", "lse", "dhidden", "dweight"}
    _close(full, ref)
    alone = E.linear_distillation_grad(h, w, ids, z, out["lse"], g, temperature=temp)
    _close(alone, R.linear(h, w, given, 0, vocab, temp, lse=out["lse"], grad_loss=g))


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_losses_of_whole_tiles(dtype):
    """Every workgroup of a full launch of the wide tiles, in each of the products."""
    rows, cols, vocab = 2048, 256, 8192
    h, w, t, g = _case(rows, cols, vocab, dtype, 5)
    _close(E.linear_cross_entropy(h, w, t, grad_loss=g), R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g))
    rows, cols, vocab = 2048, 8192, 512
    h, w, t, g = _case(rows, cols, vocab, dtype, 6)
    ids, z = _teacher(rows, 16, vocab, 7)
    _close(E.linear_distillation(h, w, ids, z, grad_loss=g, temperature=2.0),
           R.linear(h, w, R.entries(ids, z, vocab, 2.0), 0, vocab, 2.0, grad_loss=g))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [(2048, 128, 8900), (300, 2048, 8900), (2300, 8192, 300), (2300, 2048, 8900), (2300, 8192, 2100)])
def test_linear_losses_of_two_shapes_of_tiles(rows, cols, vocab, dtype):
    """A full launch of wide tiles and some middle ones behind it: of the logits, of the table's and of the hidden states' gradient;
    with longer sums, of which the middle tiles take parts."""
    h, w, t, g = _case(rows, cols, vocab, dtype, 5)
    out = E.linear_cross_entropy(h, w, t, grad_loss=g)
    _close(out, R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g))
    old = _normal(_gen(1), vocab, cols, std=1e-3, dtype=dtype)
    got = E.linear_cross_entropy_grad(h, w, t, out["lse"], g, out={"dweight": old.clone()}, accumulate=True)
    _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, lse=out["lse"], grad_loss=g, old=old))
    ids, z = _teacher(rows, 70, vocab, 7)
    _close(E.linear_distillation(h, w, ids, z, grad_loss=g, temperature=2.0),
           R.linear(h, w, R.entries(ids, z, vocab, 2.0), 0, vocab, 2.0, grad_loss=g))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [(7320, 130, 224), (3000, 896, 1283), (5000, 3000, 700)])
def test_linear_losses_of_many_rows_and_few_ids(rows, cols, vocab, dtype):
    """The table's gradient has few tiles and a long sum, of which workgroups take parts."""
    h, w, t, g = _case(rows, cols, vocab, dtype, 5)
    old = _normal(_gen(1), vocab, cols, std=1e-3, dtype=dtype)
    got = E.linear_cross_entropy(h, w, t, grad_loss=g, out={"dweight": old.clone()}, accumulate=True)
    _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g, old=old))
    lse = got["lse"]
    got = E.linear_cross_entropy_grad(h, w, t, lse, g, dtype=F32)
    _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, lse=lse, grad_loss=g))


def test_linear_pieces_with_two_shapes_of_tiles():
    """Pieces of the vocabulary after the first, of whose table's gradient the middle tiles take parts."""
    rows, cols, vocab = 40000, 1024, 26000
    h, w, t, g = _case(rows, cols, vocab, BF16, 5)
    lse = E.linear_cross_entropy(h, w, t, vocab_start=0, vocab_size=vocab)["lse"]
    got = E.linear_cross_entropy_grad(h, w, t, lse, g)
    _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, lse=lse, grad_loss=g))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [(512, 512, 4096), (2048, 128, 9000), (200, 2048, 300), (40, 128, 60000)])
def test_products_without_rounding(rows, cols, vocab, dtype):
    """Small whole numbers: every product and every sum is exact, so that logits are the plain form's to the last bit and the
    loss is off by the softmax's own few roundings only; a misplaced element cannot hide in a bound."""
    g = _gen(rows)
    h = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").to(dtype)
    w = (torch.randint(-2, 3, (vocab, cols), generator=g, device="cuda") / 64).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    x = h.double() @ w.double().t()
    ref = R.loss(x, torch.zeros_like(x), *R.targets(t, vocab), 0, vocab, 1.0)
    _close(E.linear_cross_entropy(h, w, t), ref)
    shard = E.linear_cross_entropy(h, w, t, vocab_start=0, vocab_size=vocab)
    assert torch.equal(shard["target"].double(), x.gather(1, t[:, None])[:, 0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [300, 1000])
def test_linear_shards(vocab, dtype):
    rows, cols, ranks, temp = 70, 128, 3, 2.0
    whole = vocab * ranks
    h, w, t, g = _case(rows, cols, whole, dtype, vocab)
    ids, z = _teacher(rows, 12, whole, 3)
    for given, args, more, call, grad, names in (
            (R.targets(t, whole), (t,), {}, E.linear_cross_entropy, E.linear_cross_entropy_grad, {"lse", "target"}),
            (R.entries(ids, z, whole, temp), (ids, z), dict(temperature=temp), E.linear_distillation, E.linear_distillation_grad,
             {"lse", "target", "entropy"})):
        scale = temp if more else 1.0
        parts = []
        for rank in range(ranks):
            at = dict(vocab_start=rank * vocab, vocab_size=whole, **more)
            part = w[rank * vocab:(rank + 1) * vocab]
            out = call(h, part, *args, **at)
            assert set(out) == names
            _close(out, R.linear(h, part, given, rank * vocab, whole, scale))
            parts.append(out)
        lse = torch.logsumexp(torch.stack([p["lse"] for p in parts]), 0)
        dh = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
        for rank in range(ranks):
            at = dict(vocab_start=rank * vocab, vocab_size=whole, **more)
            part = w[rank * vocab:(rank + 1) * vocab]
            out = grad(h, part, *args, lse, g, **at)
            _close(out, R.linear(h, part, given, rank * vocab, whole, scale, lse=lse, grad_loss=g))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_linear_pieces_of_the_vocabulary(dtype):
    """More than 1 GiB of the logits' gradient: it is made in pieces, whose shares of dhidden are added up."""
    rows, cols, vocab = (16384, 64, 36000) if dtype == BF16 else (8192, 64, 25000)
    h, w, t, g = _case(rows, cols, vocab, dtype, 9)
    ids, z = _teacher(rows, 4, vocab, 3)
    out = E.linear_cross_entropy(h, w, t, grad_loss=g)
    _close(out, R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g))
    out = E.linear_distillation(h, w, ids, z, grad_loss=g)
    _close(out, R.linear(h, w, R.entries(ids, z, vocab, 1.0), 0, vocab, grad_loss=g))


def test_linear_many_rows():
    """Pieces of the vocabulary whose shares of the gradient are a gigabyte each, and sums over a million rows."""
    rows, cols, vocab, chunk = 1_100_000, 64, 1000, 100_000
    h, w, t, _ = _case(rows, cols, vocab, F16, 4)
    g = torch.ones(rows, device="cuda")
    out = E.linear_cross_entropy(h, w, t, grad_loss=g, dtype=F32)
    value = bound = 0
    for i in range(0, rows, chunk):
        at = slice(i, i + chunk)
        ref = R.linear(h[at], w, R.targets(t[at], vocab), 0, vocab, grad_loss=g[at])
        v, e = ref.pop("dweight")
        # a chunk's bound has 2 U chunk times the sum of its terms' sizes, the whole sum's 2 U rows times it
        value, bound = value + v, bound + e * (rows / chunk)
        _close({k: out[k][at] for k in ref if k in out}, ref, [k for k in ref if k in out])
    R.close(out["dweight"], value, bound, "dweight")


def test_linear_table_past_32_bits():
    rows, cols, vocab = 3, 2048, 1_100_000      # 4.5 GB of bf16
    g = _gen(3)
    w = torch.empty(vocab, cols, dtype=BF16, device="cuda")
    for i in range(0, vocab, 100_000):
        w[i:i + 100_000] = _normal(g, 100_000, cols, std=0.05, dtype=BF16)
    h = _normal(g, rows, cols, dtype=BF16)
    t = torch.tensor([vocab - 1, 1_060_000, 5], device="cuda")
    x = torch.cat([h.double() @ w[i:i + 100_000].double().t() for i in range(0, vocab, 100_000)], 1)
    e = 2 * R.U * cols * torch.cat([h.abs().double() @ w[i:i + 100_000].abs().double().t() for i in range(0, vocab, 100_000)], 1)
    gl = torch.tensor([1.0, 0.5, -2.0], device="cuda")
    ref = R.loss(x, e, *R.targets(t, vocab), 0, vocab, 1.0, grad_loss=gl)
    d, e_d = ref.pop("grad")
    out = E.linear_cross_entropy(h, w, t, grad_loss=gl)
    _close(out, ref, ["loss", "lse"])
    e_d = e_d + d.abs() * (2.0 ** -8 + 16 * R.U) + 2.0 ** -120
    for i in (0, 900_000, 1_000_000):
        v, b = R.product(d[:, i:i + 100_000].t(), h.double(), BF16, e_d[:, i:i + 100_000].t())
        R.close(out["dweight"][i:i + 100_000], v, b + 8 * R.U * v.abs(), f"dweight from {i}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,vocab", [(150, 192, 400), (1100, 512, 9000), (9, 2048, 9000)])
def test_linear_gradients_added_up_and_in_32_bits(rows, cols, vocab, dtype):
    h, w, t, g = _case(rows, cols, vocab, dtype, 4)
    g = g * torch.linspace(-1, 2, rows, device="cuda")
    ref = R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g)
    out = E.linear_cross_entropy(h, w, t, grad_loss=g, dtype=F32)
    assert out["dweight"].dtype == F32
    _close(out, ref)
    for kind in {F32, dtype}:
        old = _normal(_gen(8), vocab, cols, std=0.01, dtype=kind)
        main = old.clone()
        got = E.linear_cross_entropy(h, w, t, grad_loss=g, out={"dweight": main}, accumulate=True)
        assert got["dweight"] is main
        _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=g, old=old))
        main = old.clone()
        lse = out["lse"]
        got = E.linear_cross_entropy_grad(h, w, t, lse, g, out={"dweight": main}, accumulate=True)
        _close(got, R.linear(h, w, R.targets(t, vocab), 0, vocab, lse=lse, grad_loss=g, old=old))


def test_linear_rows_not_trained_on():
    rows, cols, vocab = 70, 64, 300
    h, w, t, g = _case(rows, cols, vocab, BF16, 4)
    none = torch.full_like(t, -100)
    none[::5], none[1::5], none[2::5], none[3::5] = 2 ** 63 - 1, -2 ** 63, vocab, 2 ** 32 + 3
    out = E.linear_cross_entropy(h, w, none, grad_loss=g)
    assert not out["loss"].any() and not out["dhidden"].any() and not out["dweight"].any()
    ids, z = _teacher(rows, 5, vocab, 1)
    for i, y in ((none[:, None].expand(rows, 5).contiguous(), z), (ids, torch.full_like(z, -math.inf))):
        out = E.linear_distillation(h, w, i, y, grad_loss=g)
        assert not out["loss"].any() and not out["dhidden"].any() and not out["dweight"].any()
        R.close(out["lse"], *R.linear(h, w, R.targets(t, vocab), 0, vocab)["lse"], "lse")
    for weights in (torch.zeros_like(g), -g, g * torch.arange(rows, device="cuda") % 3):
        out = E.linear_cross_entropy(h, w, t, grad_loss=weights)
        if not weights.any():
            assert not out["dhidden"].any() and not out["dweight"].any()
        else:
            _close(out, R.linear(h, w, R.targets(t, vocab), 0, vocab, grad_loss=weights))


def test_linear_no_rows():
    w = _normal(_gen(1), 30, 64, dtype=BF16)
    h, t, g = w[:0], torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    out = E.linear_cross_entropy(h, w, t, grad_loss=g, out={"dweight": torch.full_like(w, 3)})
    assert out["loss"].shape == (0,) and out["dhidden"].shape == (0, 64) and not out["dweight"].any()
    keep = torch.full((30, 64), 2.5, device="cuda")
    out = E.linear_cross_entropy_grad(h, w, t, g, g, out={"dweight": keep}, accumulate=True)
    assert (keep == 2.5).all()
    ids = torch.empty(0, 4, dtype=torch.int64, device="cuda")
    assert E.linear_distillation(h, w, ids, ids.float())["loss"].shape == (0,)
    assert E.distillation(w[:0], ids, ids.float())["loss"].shape == (0,)


def test_linear_infinities_and_nan():
    rows, cols, vocab = 70, 64, 300
    h, w, t, g = _case(rows, cols, vocab, BF16, 4)
    t[5], t[6] = 3, 3
    bad = h.clone()
    bad[5, 7] = math.nan
    out, good = E.linear_cross_entropy(bad, w, t, grad_loss=g), E.linear_cross_entropy(h, w, t, grad_loss=g)
    others = torch.arange(rows, device="cuda") != 5
    for k in ("loss", "lse", "dhidden"):
        assert torch.isnan(out[k][5]).all() and torch.equal(out[k][others], good[k][others]), k
    assert torch.isnan(out["dweight"]).all()
    # a logit of -inf has no probability; a target there an infinite loss
    h2, w2 = h.clone(), w.clone()
    h2[:, 0], w2[:, 0] = 1.0, 0.0
    w2[3] = 0.0
    w2[3, 0] = -math.inf
    out = E.linear_cross_entropy(h2, w2, t)
    x = h2.double()[:, 1:] @ w2.double()[:, 1:].t()
    x[:, 3] = -math.inf
    ref = R.loss(x, 2 * R.U * cols * (h2.double()[:, 1:].abs() @ w2.double()[:, 1:].abs().t()), *R.targets(t, vocab), 0, vocab, 1.0)
    _close(out, ref)
    assert torch.isinf(out["loss"][5])
    w2[3, 0] = math.inf
    out = E.linear_cross_entropy(h2, w2, t)
    assert torch.isnan(out["lse"]).all()


def test_linear_shapes_views_and_broadcast_rows():
    rows, cols, vocab = 12, 128, 300
    h, w, t, g = _case(rows, cols, vocab, BF16, 4)
    flat = E.linear_cross_entropy(h, w, t, grad_loss=g)
    out = E.linear_cross_entropy(h.view(3, 4, cols), w, t.view(3, 4), grad_loss=g.view(3, 4))
    assert out["loss"].shape == (3, 4) and out["dhidden"].shape == (3, 4, cols)
    assert all(torch.equal(out[k].reshape(flat[k].shape), flat[k]) for k in flat)
    wide = torch.full((vocab, 3 * cols), math.nan, dtype=BF16, device="cuda")
    wide[:, cols:2 * cols] = w
    out = E.linear_cross_entropy(h, wide[:, cols:2 * cols], t, grad_loss=g)      # rows in order, far apart
    assert all(torch.equal(out[k], flat[k]) for k in flat)
    same = h[:1].expand(rows, cols)
    _close(E.linear_cross_entropy(same, w, t, grad_loss=g), R.linear(same, w, R.targets(t, vocab), 0, vocab, grad_loss=g))
    ids, z = _teacher(rows, 6, vocab, 1)
    a = E.linear_distillation(h.view(3, 4, cols), w, ids.view(3, 4, 6), z.view(3, 4, 6), grad_loss=g.view(3, 4))
    b = E.linear_distillation(h, w, ids, z, grad_loss=g)
    assert a["loss"].shape == (3, 4) and all(torch.equal(a[k].reshape(b[k].shape), b[k]) for k in b)
    space = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    c = E.linear_distillation(h, w, ids, z, grad_loss=g, workspace=space)
    assert all(torch.equal(c[k], b[k]) for k in b)


def _agrees(value, grad, v):
    """A directional derivative by differences and the gradient's."""
    want = float((grad.double() * v).sum())
    assert abs(value - want) <= 1e-4 * (abs(want) + float((grad.double().abs() * v.abs()).sum()) * 1e-2), (value, want)


@pytest.mark.parametrize("temp", [1.0, 2.5])
def test_gradients_against_differences(temp):
    """The 64-bit loss by central differences of step 1e-5: its third derivative is below 10 here, so that they are good to 1e-9."""
    rows, cols, vocab = 9, 24, 50
    h, w, t, g = _case(rows, cols, vocab, F32, 4)
    ids, z = _teacher(rows, 5, vocab, 3)
    gl = _normal(_gen(2), rows)

    def total(a, b):
        x = (a @ b.t()) / temp
        zero = torch.zeros_like(x)
        return (R.loss(x, zero, *R.entries(ids, z, vocab, temp), 0, vocab, temp)["loss"][0] * gl.double()).sum()

    out = E.linear_distillation(h, w, ids, z, temperature=temp, grad_loss=gl)
    a, b = h.double(), w.double()
    for k, seed in (("dhidden", 1), ("dweight", 2)):
        v = _normal(_gen(seed), *out[k].shape).double()
        s = 1e-5 * v
        if k == "dhidden":
            d = total(a + s, b) - total(a - s, b)
        else:
            d = total(a, b + s) - total(a, b - s)
        _agrees(float(d) / 2e-5, out[k], v)
    l = (h @ w.t()).contiguous()
    grad = E.distillation(l, ids, z, temperature=temp, grad_loss=gl)["grad"]
    v = _normal(_gen(5), rows, vocab).double()

    def of(x):
        return (R.loss(x / temp, torch.zeros_like(x), *R.entries(ids, z, vocab, temp), 0, vocab, temp)["loss"][0] * gl.double()).sum()

    _agrees(float(of(l.double() + 1e-5 * v) - of(l.double() - 1e-5 * v)) / 2e-5, grad, v)


# ---------------------------------------------------------------- distillation of logits

WIDTHS = [1, 3, 8, 64, 100, 513, 2048, 2051, 6400, 8193, 20000, 32768, 32775, 51200, 65536, 65537, 100003]


def _check_distill(l, ids, z, temp, g, **kw):
    cols = l.shape[-1]
    ref = R.distillation(l, ids, z, 0, cols, temp, grad_loss=g)
    out = E.distillation(l, ids, z, temperature=temp)
    assert set(out) == {"loss", "lse"}
    _close(out, ref)
    full = E.distillation(l, ids, z, temperature=temp, grad_loss=g, **kw)
    assert set(full) == {"loss", "lse", "grad"}
    _close(full, ref)
    alone = E.distillation_grad(l, ids, z, out["lse"], g, temperature=temp)
    R.close(alone, *R.distillation(l, ids, z, 0, cols, temp, lse=out["lse"], grad_loss=g)["grad"], "grad alone")
    return full


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_distillation_widths(cols, dtype):
    for rows, top, temp in ((1, 1, 1.0), (5, 8, 2.0), (70, 33, 0.7)) if cols < 10000 else ((1, 64, 4.0), (3, 200, 1.0)):
        g = _gen(cols + rows)
        l = _normal(g, rows, cols, std=2.5, dtype=dtype)
        ids, z = _teacher(rows, top, cols, rows, dtype if rows == 5 else F32, torch.int32 if rows == 5 else torch.int64)
        gl = _normal(g, rows)
        full = _check_distill(l, ids, z, temp, gl)
        odd = E.distillation(_odd(l), ids, z, temperature=temp, grad_loss=gl, out={"grad": _odd(l, 2, 1)})
        assert all(torch.equal(odd[k], full[k]) for k in full)
        same = l.clone()
        put = E.distillation(same, ids, z, temperature=temp, grad_loss=gl, out={"grad": same})
        assert put["grad"] is same and all(torch.equal(put[k], full[k]) for k in full)
        same = l.clone()
        assert torch.equal(E.distillation_grad(same, ids, z, full["lse"], gl, temperature=temp, out=same),
                           E.distillation_grad(l, ids, z, full["lse"], gl, temperature=temp))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [9, 1000, 6400, 40000, 70000])
def test_distillation_shards(cols, dtype):
    rows, top, ranks, temp = 6, 40, 3, 2.0
    whole = cols * ranks
    g = _gen(cols)
    l, gl = _normal(g, rows, whole, std=2.5, dtype=dtype), _normal(g, rows)
    ids, z = _teacher(rows, top, whole, 3)
    lse = []
    for rank in range(ranks):
        part = l[:, rank * cols:(rank + 1) * cols]
        out = E.distillation(part, ids, z, temperature=temp, vocab_start=rank * cols, vocab_size=whole)
        assert set(out) == {"lse", "target", "entropy"}
        _close(out, R.distillation(part, ids, z, rank * cols, whole, temp))
        lse.append(out["lse"])
    lse = torch.logsumexp(torch.stack(lse), 0)
    for rank in range(ranks):
        part = l[:, rank * cols:(rank + 1) * cols]
        out = E.distillation_grad(part, ids, z, lse, gl, temperature=temp, vocab_start=rank * cols, vocab_size=whole)
        R.close(out, *R.distillation(part, ids, z, rank * cols, whole, temp, lse=lse, grad_loss=gl)["grad"], "grad")


@pytest.mark.parametrize("cols", [500, 5000, 40000, 70000])
def test_distillation_edges(cols):
    g = _gen(cols)
    rows, top = 9, 6
    l, gl = _normal(g, rows, cols, std=2.0), _normal(g, rows)
    ids = torch.randint(0, cols, (rows, top), generator=g, device="cuda")
    z = _normal(g, rows, top)
    ids[0] = -100                                              # no id
    z[1] = -math.inf                                           # no mass
    ids[2] = ids[2, 0]                                         # one id six times
    z[3, 1:4] = -math.inf
    l[4, ids[4, 0]] = -math.inf                                # a mass where the student has none
    z[4, 0] = 1.0
    l[5, ids[5, 0]] = -math.inf                                # and none where the teacher has none either
    z[5, 0] = -math.inf
    l[6] = -math.inf                                           # no logit
    ids[7] = torch.tensor([2 ** 63 - 1, -2 ** 63, cols, -1, 7, 2 ** 32 + 7], device="cuda")
    out = _check_distill(l, ids, z, 2.0, gl)
    assert out["loss"][0] == 0 and out["loss"][1] == 0 and out["loss"][4] == math.inf and out["loss"][6] == math.inf
    assert not out["grad"][0].any() and not out["grad"][1].any() and not out["grad"][6].any()
    for change in ("logit", "teacher"):
        l2, z2 = l.clone(), z.clone()
        if change == "logit":
            l2[3, 11] = math.nan
        else:
            z2[3, 0] = math.nan
        bad = E.distillation(l2, ids, z2, temperature=2.0, grad_loss=gl)
        assert torch.isnan(bad["loss"][3])
        others = torch.arange(rows, device="cuda") != 3
        assert all(torch.equal(bad[k][others], out[k][others]) for k in out)


# ---------------------------------------------------------------- streams, graphs, together

def _calls():
    h, w, t, g = _case(130, 128, 700, BF16, 3)
    ids, z = _teacher(130, 9, 700, 3)
    l = (h @ w.t()).contiguous()
    lse = E.cross_entropy(l, t)["lse"]
    return {
        "cross entropy": lambda: E.linear_cross_entropy(h, w, t, grad_loss=g),
        "cross entropy grad": lambda: E.linear_cross_entropy_grad(h, w, t, lse, g),
        "linear distillation": lambda: E.linear_distillation(h, w, ids, z, temperature=2.0, grad_loss=g),
        "distillation": lambda: E.distillation(l, ids, z, temperature=2.0, grad_loss=g),
        "distillation grad": lambda: {"grad": E.distillation_grad(l, ids, z, lse, g)},
        "float32": lambda: E.linear_cross_entropy(h.float(), w.float(), t, grad_loss=g),
    }


@pytest.mark.parametrize("name", ["cross entropy", "cross entropy grad", "linear distillation", "distillation", "distillation grad",
                                  "float32"])
def test_other_streams_and_graphs(name):
    call = _calls()[name]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call()
    s.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        for v in held.values():
            v.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[k], want[k]) for k in want)
        eager = call()
        assert all(torch.equal(eager[k], want[k]) for k in want)


def test_graphs_and_calls_that_share_a_workspace():
    a, b = _case(130, 128, 700, BF16, 3), _case(90, 64, 900, BF16, 5)
    space = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    wants, graphs = [], []
    for h, w, t, g in (a, b):
        wants.append(E.linear_cross_entropy(h, w, t, grad_loss=g))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            held = E.linear_cross_entropy(h, w, t, grad_loss=g, workspace=space)
        graphs.append((graph, held))
    space.fill_(255)
    for _ in range(3):
        for (graph, held), want in zip(graphs, wants):
            graph.replay()
        torch.cuda.synchronize()
        for (graph, held), want in zip(graphs, wants):
            assert all(torch.equal(held[k], want[k]) for k in want)


def test_written_tensors_count_as_modified_and_graphs_are_refused():
    h, w, t, g = _case(10, 64, 100, F32, 3)
    main = torch.zeros(100, 64, device="cuda")
    before = main._version
    E.linear_cross_entropy(h, w, t, grad_loss=g, out={"dweight": main}, accumulate=True)
    assert main._version > before
    leaf = w.clone().requires_grad_()
    with pytest.raises(E.EchoError, match="requires grad"):
        E.linear_cross_entropy(h, leaf, t)
    with torch.no_grad():
        E.linear_cross_entropy(h, leaf, t)


def test_teachers_that_repeat_themselves():
    """An id in every place, ids in pairs, an id of which one entry has no mass: the masses of an id add up in its first entry."""
    rows, cols, vocab = 5, 64, 700
    h, w, _, g = _case(rows, cols, vocab, F32, 1)
    for top in (2, 65, 130, 1024):
        gen = _gen(top)
        ids = torch.randint(0, vocab, (rows, top), generator=gen, device="cuda")
        z = _normal(gen, rows, top)
        ids[0] = 7
        ids[1, 1::2] = ids[1, 0::2][:ids[1, 1::2].numel()]
        ids[2, top // 2:] = ids[2, 0]
        z[2, 0] = -math.inf
        ids[3] = torch.arange(top, device="cuda") % 3
        ids[4, ::2] = -1
        given = R.entries(ids, z, vocab, 1.0)
        _close(E.linear_distillation(h, w, ids, z, grad_loss=g), R.linear(h, w, given, 0, vocab, grad_loss=g))
        l = (h @ w.t()).contiguous()
        _close(E.distillation(l, ids, z, grad_loss=g), R.distillation(l, ids, z, 0, vocab, 1.0, grad_loss=g))
        wide = torch.cat([l, _normal(gen, rows, 9000)], 1)      # tiles with cells, not rows of parts
        assert wide.shape[1] == vocab + 9000
        _close(E.distillation(wide, ids, z, grad_loss=g), R.distillation(wide, ids, z, 0, vocab + 9000, 1.0, grad_loss=g))
    rows, cols, vocab = 1030, 64, 6000
    h, w, _, g = _case(rows, cols, vocab, BF16, 2)
    ids, z = _teacher(rows, 300, vocab, 4)
    ids[:, 100:200] = ids[:, :100]
    _close(E.linear_distillation(h, w, ids, z, grad_loss=g), R.linear(h, w, R.entries(ids, z, vocab, 1.0), 0, vocab, grad_loss=g))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step_with_the_head_in_one_call(dtype):
    """The operators together, against the same step with a library product for the head: the loss, and gradients that differ by
    the roundings of logits and their gradient to the activations' type alone."""
    from workloads import measured

    g = _gen(7)
    vocab, cols, tokens = 600, 128, 96
    table = _normal(g, vocab, cols, std=0.3, dtype=dtype)
    norms = [(torch.ones(cols, device="cuda", dtype=dtype), torch.zeros(cols, device="cuda", dtype=dtype)) for _ in range(3)]
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets[::6] = -100
    a = measured.training_step(ids, targets, table, norms)
    b = measured.training_step(ids, targets, table, norms, fused=True)
    unit = R.UNIT[dtype]
    # logits of up to |l| < 16 are rounded to their type in the one and not in the other; so are the gradients
    assert abs(float(a["loss"] - b["loss"])) <= 32 * unit + 1e-5
    for x, y in [(a["table"], b["table"])] + [(x, y) for m, n in zip(a["norms"], b["norms"]) for x, y in zip(m, n)]:
        assert float((x - y).norm()) <= (64 * unit + 1e-5) * float(x.norm())
    again = measured.training_step(ids, targets, table, norms, fused=True)
    assert torch.equal(again["table"], b["table"])
    # a teacher beside the targets: the loss is their sum, and so are the gradients
    tid, z = _teacher(tokens, 8, vocab, 3)
    c = measured.training_step(ids, targets, table, norms, fused=True, teacher=(tid, z, 2.0))
    h = measured.training_step(ids, torch.full_like(targets, -100), table, norms, fused=True, teacher=(tid, z, 2.0))
    assert abs(float(c["loss"] - b["loss"] - h["loss"])) <= 1e-4 * (1 + abs(float(c["loss"])))
    assert float((c["table"] - b["table"] - h["table"]).norm()) <= (64 * unit + 1e-5) * float(c["table"].norm())
