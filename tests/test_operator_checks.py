"""The comparison of the experts' outputs rejects what it is there for: fewer bits, a k tile, a column tile, an expert, an element."""
import pytest
import torch
import operator_checks as K

# (T, E, k, d, ff): the shapes that the outputs of the kernels are checked at
SHAPES = [(1, 8, 2, 256, 704), (7, 8, 2, 512, 1344), (16, 64, 8, 128, 72), (31, 5, 3, 200, 136), (64, 16, 4, 320, 200), (100, 8, 2, 768, 1088),
          (100, 5, 4, 520, 264), (257, 9, 2, 136, 264), (900, 6, 3, 328, 712), (1500, 5, 4, 520, 264), (60, 4, 2, 1032, 5480), (1200, 2, 2, 1032, 5480)]
WIDE = (3, 2, 2, 4096, 14336)


def _case(shape, half):
    T, E, k, d, ff = shape
    g = torch.Generator().manual_seed(T + d)
    dt = torch.bfloat16 if half else torch.float32

    def normal(*s, std=1.0):
        return torch.empty(s).normal_(0.0, std, generator=g).to(dt).double()

    mats = (normal(E, ff, d, std=d ** -0.5), normal(E, ff, d, std=d ** -0.5), normal(E, d, ff, std=ff ** -0.5))
    ids = torch.rand(T, E, generator=g).argsort(1)[:, :k]
    return normal(T, d), ids, torch.rand(T, k, generator=g).double() + 0.1, mats


def _run(x, ids, w, mats, half, cut=None):
    """The experts in the arithmetic of a mode: float32 products and sums; float16 operands.  cut: the first column behind a down
    product's left-out k tile of 32."""
    y = torch.zeros(x.shape)
    for e in range(mats[0].shape[0]):
        row, place = torch.nonzero(ids == e, as_tuple=True)
        if row.numel():
            a, b, c = (m[e].float() for m in mats)
            xe = x[row].float()
            g = xe @ a.T
            hid = g / (1 + torch.exp(-g)) * (xe @ b.T)
            if half:
                hid = hid.half().float()
            if cut:
                hid[:, max(cut - 32, 0):cut] = 0
            y.index_add_(0, row, w[row, place].float()[:, None] * (hid @ c.T))
    return y.bfloat16() if half else y


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("shape", SHAPES + [WIDE])
def test_what_is_wrong_is_rejected(shape, half):
    T, E, k, d, ff = shape
    x, ids, w, mats = _case(shape, half)
    ref, expected = K.experts(x, ids, w, *mats, half)
    y = _run(x, ids, w, mats, half)
    assert K.worst_tile(y, ref, expected, half) <= 1.0

    def rejected(v):
        return K.worst_tile(v, ref, expected, half) > 1.0

    if not half:
        low = [m.bfloat16().double() for m in mats]
        assert rejected(_run(x.bfloat16().double(), ids, w, low, half))
        assert rejected(y.half().float()) and rejected(y.bfloat16().float())
    assert rejected(_run(x, ids, w, mats, half, cut=ff // 2))
    cut = y.clone()
    cut[:, d // 2 // 16 * 16:][:, :16] = 0
    assert rejected(cut)
    if E > 1:                                             # the first row's first expert for another
        other = ids.clone()
        other[0, 0] = next(e for e in range(E) if e not in ids[0]) if k < E else ids[0, 1]
        assert rejected(_run(x, other, w, mats, half))
    one = y.clone()
    r, c = divmod(int(ref.abs().argmax()), d)
    one[r, c] = 0
    assert rejected(one)
