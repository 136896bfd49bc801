"""Every variant of the training-step operators' kernels on the GPU against the plain 64-bit forms: each width's, a team that
works on several rows in turn, and launches whose workgroups go round more than once."""
from __future__ import annotations

import pytest
import torch

import paper_2412_12487_amd as E
from tests import opsref as R
from tests import opsvariants as V

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, mean=0.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


def _compare(out, ref, at=slice(None)):
    for k, (v, e) in ref.items():
        if k in out:
            R.close(out[k][at] if out[k].dim() == v.dim() else out[k].reshape(v.shape), v, e, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", V.NORM_WIDTHS)
def test_layer_norm_variants(cols, dtype):
    g = _gen(cols)
    for rows, wide, residual in ((6, False, True), (9, True, False)):
        x, r = _normal(g, rows, cols, std=1.5, mean=0.7, dtype=dtype), _normal(g, rows, cols, dtype=dtype) if residual else None
        wt = F32 if wide else dtype
        w, b = _normal(g, cols, std=0.2, mean=1.0, dtype=wt), _normal(g, cols, std=0.3, dtype=wt)
        out = E.layer_norm(x, w, b, residual=r)
        h = x if r is None else (x.float() + r.float()).to(dtype)
        assert r is None or torch.equal(out["sum"], h)
        _compare(out, R.layer_norm(h, w, b, 1e-5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", V.NORM_WIDTHS)
def test_layer_norm_grad_variants_over_several_rows_a_team(cols, dtype):
    """Every team has three rows at least, and some a fourth: both rows in flight are fetched anew, and the exchange
    between its wavefronts changes its buffer twice."""
    variant, _ = V.norm_grad(cols, 4 if dtype == F32 else 2)
    most = (512 if cols <= 2048 else 256) * V.teams(variant)      # rows of one turn, at most
    rows = 3 * most + 77
    g = _gen(cols + 1)
    x, dy, dr = (_normal(g, rows, cols, std=s, mean=m, dtype=dtype) for s, m in ((1.5, 0.3), (0.5, 0.05), (0.5, 0.0)))
    w = _normal(g, cols, std=0.2, mean=1.0, dtype=dtype)
    s = E.layer_norm(x, w)
    out = E.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], grad_residual=dr, dtype=F32)
    _compare(out, R.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], dr))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", V.LOSS_WIDTHS)
def test_cross_entropy_variants(cols, dtype):
    g = _gen(cols + 2)
    l, t, gl = _normal(g, 5, cols, std=2.5, dtype=dtype), torch.randint(0, cols, (5,), generator=g, device="cuda"), _normal(g, 5)
    t[0], t[1], t[3] = cols - 1, -100, 0
    want = R.cross_entropy(l, t, 0, cols, grad_loss=gl)
    _compare(E.cross_entropy(l, t), want)
    out = E.cross_entropy(l, t, grad_loss=gl)
    _compare(out, want)
    same = l.clone()
    again = E.cross_entropy(same, t, grad_loss=gl, out={"grad": same})
    assert all(torch.equal(again[k], out[k]) for k in out)


ROUND = 1 << 20      # workgroups of a launch, at most


def _windows(g, rows, cols, dtype, std):
    """rows x cols, row r beginning 8 elements after row r - 1: all of them different, in little memory."""
    return torch.as_strided(_normal(g, rows * 8 + cols, std=std, dtype=dtype), (rows, cols), (8, 1))


def _ends(rows, first):
    """The first rows, and those around the first that a workgroup takes in its second turn to the end."""
    return torch.cat([torch.arange(0, 40), torch.arange(first - 40, rows)]).cuda()


@pytest.mark.parametrize("cols", [3, 24, 1032, 6152])
def test_layer_norm_of_more_rows_than_a_launch_has_teams(cols):
    variant, _ = V.norm(cols, 2)
    first = ROUND * V.teams(variant)
    rows = first + 70
    g = _gen(cols)
    x = _windows(g, rows, cols, BF16, 1.5)
    w, b = _normal(g, cols, std=0.2, mean=1.0, dtype=BF16), _normal(g, cols, dtype=BF16)
    out = E.layer_norm(x, w, b)
    at = _ends(rows, first)
    _compare({k: v[at] for k, v in out.items()}, R.layer_norm(x[at], w, b, 1e-5))
    if cols == 3:
        d = E.layer_norm_grad(out["y"], x, w, out["mean"], out["rstd"])
        ref = R.layer_norm_grad(out["y"][at], x[at], w, out["mean"][at], out["rstd"][at])
        R.close(d["dx"][at], *ref["dx"], "dx")


@pytest.mark.parametrize("cols", [3, 24, 2056, 16392, 40968])
def test_cross_entropy_of_more_rows_than_a_launch_has_teams(cols):
    variant, _ = V.loss(cols, 2)
    first = ROUND * V.teams(variant)
    rows = first + 70
    g = _gen(cols)
    l = _windows(g, rows, cols, BF16, 2.5)
    t = torch.randint(0, cols, (rows,), generator=g, device="cuda", dtype=torch.int32)
    gl = _normal(g, rows)
    at = _ends(rows, first)
    ref = R.cross_entropy(l[at], t[at], 0, cols, grad_loss=gl[at])
    _compare({k: v[at] for k, v in E.cross_entropy(l, t).items()}, ref)
    if cols <= 2056:
        out = E.cross_entropy(l, t, grad_loss=gl)
        _compare({k: v[at] for k, v in out.items()}, ref)
        ref = R.cross_entropy(l[at], t[at], 0, cols, lse=out["lse"][at], grad_loss=gl[at])
        R.close(E.cross_entropy_grad(l, t, out["lse"], gl)[at], *ref["grad"], "grad alone")


def test_embedding_of_more_tokens_than_a_launch_has_wavefronts():
    rows = 4 * ROUND + 70
    g = _gen(5)
    w = _normal(g, 1000, 24, dtype=BF16)
    ids = torch.randint(0, 1000, (rows,), generator=g, device="cuda")
    assert torch.equal(E.embedding(ids, w, 1.0), w[ids])
    dy = torch.ones(rows, 24, dtype=BF16, device="cuda")
    out = E.embedding_grad(ids, dy, 1000, dtype=F32)      # sums of ones: exact
    assert torch.equal(out, torch.bincount(ids, minlength=1000).float()[:, None].expand(1000, 24))
