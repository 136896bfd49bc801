"""The output head's losses and distillation at the calls that tests/test_gpu_head.py does not make, against 64 bits: every
statistic asked for together, shards by tiles."""
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
