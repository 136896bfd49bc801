"""Which variant of a training-step operator's kernel a row's width selects, as the sources' ladders say, and widths that
together reach every one.  A variant is (lanes of a team, elements a lane); CUT rows are not whole 16-byte pieces."""
from __future__ import annotations

NORM = [(64, 8), (64, 16), (256, 8), (256, 16), (256, 24), (512, 16), (512, 24), (512, 32)]
GRAD = [(64, 8), (64, 16), (256, 8), (512, 8), (768, 8)]           # then, by whole or cut rows and element size:
GRAD_CUT, GRAD_WHOLE = [(512, 16), (512, 24)], [(1024, 8), (768, 16)]
GRAD_LAST = {2: (1024, 16), 4: (512, 32)}
LOSS = [(64, 8), (64, 32), (256, 32), (512, 32), (1024, 32), (1024, 40), (1024, 48), (1024, 64)]


def pick(ladder, cols):
    return next((v for v in ladder if cols <= v[0] * v[1]), None)


def norm(cols, size):
    """(variant or None for the kernel of wide and tiny rows, cut)"""
    n = 16 // size
    return (None if cols < n else pick(NORM, cols)), cols % n != 0


def norm_grad(cols, size):
    n = 16 // size
    cut, whole = cols % n != 0, cols - cols % n
    ladder = GRAD + (GRAD_CUT if cut else GRAD_WHOLE + [GRAD_LAST[size]])
    return (pick(ladder, whole) if whole else None), cut


def loss(cols, size):
    n = 16 // size
    return (None if cols < n else pick(LOSS, cols)), cols % n != 0


def teams(variant):
    """Rows that a workgroup works on at a time."""
    return max(1, 256 // variant[0]) if variant else 1


# both sides of every threshold, whole pieces and cut rows of either element size
NORM_WIDTHS = [3, 5, 101, 104, 512, 517, 904, 1021, 1024, 1027, 1501, 2040, 2048, 2051, 4091, 4096, 4099, 5003, 5120, 6139, 6144, 6145,
               7001, 8184, 8191, 8195, 10001, 10400, 12280, 12291, 12299, 15001, 16376, 16381, 16388, 20000, 20003]
LOSS_WIDTHS = [3, 5, 101, 104, 512, 515, 1201, 2048, 2053, 5000, 5003, 8192, 8195, 16381, 16384, 20001, 20008, 30003, 32768, 32771,
               40000, 40963, 40968, 45003, 45056, 48001, 49152, 49155, 52003, 65533, 65536, 65541, 65544]
