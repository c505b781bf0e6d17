"""Whether an output of the experts is what rounding alone leaves of the definition, tile by tile.

The worst-case bound of operator_math.experts adds every rounding of sums that are thousands of terms long at its largest, so that it is
wider than the result itself at wide experts.  Here roundings are independent errors: a float32 sum of n terms is off by at most
2^-24 sqrt(n) of the root of its terms' squares (a partial sum of i of them has the size sqrt(i / n) of that root, a rounding a variance
of a third of its half step's square: sqrt(n / 6), so 2.4 times less), a product of float16 by 2^-11, and the errors of one tile of 16 x 16
elements are compared by their root mean square: at most 4 times what they should be, and a half step of the result's own rounding.
One wrong element of a tile is a sixteenth of its root mean square, and so far out."""
import torch
from operator_math import B16, F32, H16, TINY16


def experts(x, ids, weights, wg, wu, w2, half, mats=None):
    """float64 -> (y, root mean square error to expect of every element).  wg, wu, w2 [E, ..]; or mats(e) -> the three of one expert."""
    d = x.shape[1]
    y, var, size = (torch.zeros_like(x) for _ in range(3))
    low, ff = TINY16 if half else 0.0, 0
    E = wg.shape[0] if mats is None else int(ids.max()) + 1
    for e in range(E):
        row, place = torch.nonzero(ids == e, as_tuple=True)
        if not row.numel():
            continue
        a, b, c = (wg[e], wu[e], w2[e]) if mats is None else mats(e)
        ff = a.shape[0]
        xe, w = x[row], weights[row, place][:, None]
        g, u = xe @ a.T, xe @ b.T
        x2 = xe * xe

        def sum_error2(m):                                # of x m^T
            m2 = m * m
            return (d + 2) * F32 ** 2 * (x2 @ m2.T) + low ** 2 * (x2.sum(1, keepdim=True) + m2.sum(1))

        s = g * torch.sigmoid(g)
        hid = s * u
        dh2 = (1.1 * u) ** 2 * sum_error2(a) + s ** 2 * sum_error2(b) + (8 * F32 * hid) ** 2
        if half:
            dh2 = dh2 + (H16 * hid) ** 2 + TINY16 ** 2
        c2, h2 = c * c, hid * hid
        y.index_add_(0, row, w * (hid @ c.T))
        var.index_add_(0, row, w * w * (dh2 @ c2.T + low ** 2 * (h2.sum(1, keepdim=True) + c2.sum(1))))
        size.index_add_(0, row, w * w * (h2 @ c2.T))
    return y, torch.sqrt(var + (ff + ids.shape[1] + 8) * F32 ** 2 * size)


def _tiles(v):
    """Root mean squares over the tiles of 16 x 16 elements, what lies behind the edges left out."""
    T, d = v.shape
    p = torch.nn.functional.pad(v * v, (0, -d % 16, 0, -T % 16))
    n = torch.nn.functional.pad(torch.ones_like(v), (0, -d % 16, 0, -T % 16))
    return torch.sqrt(torch.nn.functional.avg_pool2d(p[None], 16)[0] / torch.nn.functional.avg_pool2d(n[None], 16)[0])


def worst_tile(y, ref, expected, half):
    """The largest share of its bound that a tile's error has: up to 1 is right."""
    if not torch.isfinite(y).all():
        return float("inf")
    step = B16 if half else F32
    return float((_tiles(y.double() - ref) / (step * _tiles(ref) + 4 * _tiles(expected) + 1e-38)).max())
