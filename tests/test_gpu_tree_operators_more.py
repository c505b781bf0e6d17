"""More of the operators of a round of drafted trees: scores at the ends of float32, plans and variants that larger calls reach."""
import numpy as np
import pytest
import torch
import tree_math as M
from test_gpu_tree_operators import DEV, TYPES, Batch, _check_logits, _ints, _logits_case, _ops

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ scores at the ends of float32
# One batch for each kernel: few rows (one or two tiles), shared keys (64, 128, 256 rows), each whole and split.
ENDS = [([40, 9], [3, 1], 2, 2, 64, 8), ([3000], [2], 2, 1, 128, 16), ([70, 33], [5, 5], 10, 2, 64, 16), ([2500, 8], [9, 6], 6, 2, 128, 32), ([90], [40], 1, 1, 64, 8),
        ([1900], [25], 4, 2, 128, 16), ([60, 2], [50, 40], 4, 2, 64, 32), ([2100], [70], 3, 3, 128, 64), ([100], [100], 4, 2, 64, 16), ([4000], [60], 12, 3, 128, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** 9, -2.0 ** 9, 2.0 ** 40, 2.0 ** 126, 2.0 ** -119, 0.75 * 2.0 ** -117, -2.0 ** -95, 2.0 ** -86, 1.0])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh, page", ENDS)
def test_scores_at_the_ends_of_float32(dtype, scale, lens, nodes, H, KVH, dh, page):
    """Products q.k of a 2^118 with a in +-[1, 2) at steps of 2^-7.  Scales of 2^9 put the scores up to the largest float32, larger ones beyond it: the largest of a
    row takes all of the weight, ties share it, as from scores of 2^24 on.  With 2^-119 they are ordinary ones, of which each row's largest and others have weights."""
    b = Batch(sum(lens) + dh, dtype, lens, nodes, H, KVH, dh, page)
    steps = torch.randint(0, 128, b.keys.shape[:-1], generator=b.g).to(DEV)
    sign = (torch.randint(0, 2, b.keys.shape[:-1], generator=b.g) * 2 - 1).to(DEV)
    if lens[0] % 20:                                      # all of one sign: every score lies at one end
        sign[:] = 1 if lens[0] % 3 else -1
    b.keys.zero_()
    b.keys[..., 0] = (sign * (1 + steps / 128.0) * 2.0 ** 58).to(b.dtype)
    b.q.zero_()
    b.q[:, ::dh] = (torch.randint(0, 2, (b.T, H), generator=b.g).to(DEV) * 2 - 1) * 2.0 ** 60
    for visible in (None, b.seen()):
        y = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=visible, scale=scale).double().cpu().reshape(b.T, H, dh)
        # The products are exact, so a weight has the roundings of its argument: with the smallest scales, |s| < 6 and a span below 17.4 in base 2, of which the scale's
        # two roundings are 2^-24 and 2^-25, and two roundings of 2^-20, together below 2^-18 of the weight; the exponential's 2^-22 are in it.  Two bf16: 2^-16.  Weights enter
        # twice, above and below; a sum of n of them has n roundings, twice; the result its own
        want, _, mine = M.attend(b.keys[0], b.values[0], b.table, b.lens, b.first, visible, b.q.reshape(b.T, H, dh), scale, b.dtype == torch.bfloat16)
        half = b.dtype == torch.bfloat16
        n = max(l + c for l, c in zip(lens, nodes))
        wide = float(b.values.abs().max())
        bound = (2 * (2.0 ** -16 if half else 0.0) + 2 * 2.0 ** -18 + (2 * n + 16) * M.F32) * wide + (M.B16 if half else M.F32) * want.abs()
        good = bool(mine.all() and ((y - want).abs() <= bound).all())
        assert good, float((y - want).abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh, page", ENDS)
def test_scores_around_two_to_the_24(dtype, lens, nodes, H, KVH, dh, page):
    """Scores of ln 2 (2^24 + j), j even from -12 to 12: the largest of a block, a wave or a share lies on either side of the bound from which weights are made otherwise."""
    b = Batch(sum(lens) + dh, dtype, lens, nodes, H, KVH, dh, page)
    b.keys.zero_()
    b.keys[..., 0] = 2.0 ** 12
    level = 2.0 * torch.randint(-6, 7, b.keys.shape[:-1], generator=b.g)
    level = torch.where(torch.rand(level.shape, generator=b.g) < 0.9, level.clamp(max=-4), level)      # (the large ones are rare)
    b.keys[..., 1] = level.to(DEV).to(b.dtype)
    b.q.zero_()
    b.q[:, ::dh], b.q[:, 1::dh] = 2.0 ** 12, 1.0
    scale = float(np.float32(np.log(2.0)))
    half = b.dtype == torch.bfloat16
    for visible in (None, b.seen()):
        y = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=visible, scale=scale).double().cpu().reshape(b.T, H, dh)
        want, _, mine = M.attend(b.keys[0], b.values[0], b.table, b.lens, b.first, visible, b.q.reshape(b.T, H, dh), scale, half)
        # exponents span 24: two roundings of 2^-20 each for a weight and for each of at most 12 rescalings; weights enter twice
        n = max(l + c for l, c in zip(lens, nodes))
        bound = (2 * (2.0 ** -16 if half else 0.0) + 2 * 26 * 2.0 ** -20 + (2 * n + 16) * M.F32) * float(b.values.abs().max()) + (M.B16 if half else M.F32) * want.abs()
        good = bool(mine.all() and ((y - want).abs() <= bound).all())
        assert good, float((y - want).abs().max())
