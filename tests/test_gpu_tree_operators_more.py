"""More of the operators of a round of drafted trees: scores at the ends of float32, plans and variants that larger calls reach."""
import numpy as np
import pytest
import torch
import tree_math as M
from test_gpu_tree_operators import DEV, TYPES, Batch, _check_logits, _ints, _logits_case, _ops

pytestmark = pytest.mark.gpu


def _exact(b, visible=None, scale=None):
    """tree_math.attend with matrix products in float64 on the GPU, a sequence and a KV head at a time; -> y, bound [T, H, dh]."""
    scale = b.dh ** -0.5 if scale is None else scale
    half, F, INF = b.dtype == torch.bfloat16, M.F32, float("inf")
    lens, first, G, t = b.lens.tolist(), b.first.tolist(), b.H // b.KVH, b.table.long()
    y, bounds = (torch.zeros(b.T, b.KVH, G, b.dh, dtype=torch.float64, device=DEV) for _ in range(2))
    for s, l in enumerate(lens):
        n = first[s + 1] - first[s]
        if n == 0:
            continue
        slots = torch.arange(min(l + n, b.table.shape[1] * b.page), device=DEV)
        pages = t[s, slots // b.page]
        there = (pages >= 0) & (pages < b.keys.shape[1])
        pages = torch.where(there, pages, 0)
        node, j = torch.arange(n, device=DEV)[:, None], slots[None] - l
        rows = slice(first[s], first[s + 1])
        if visible is None:
            seen = j <= node
        else:
            w = visible[rows].shape[1]
            word = visible[rows].gather(1, (j.clamp(min=0) // 64).clamp(max=w - 1).expand(n, -1))
            seen = (j < 0) | ((j < 64 * w) & ((word >> (j.clamp(min=0) % 64)) & 1 == 1))
        seen = (seen & there).repeat_interleave(G, 0)                     # [n G, slots]
        for h in range(b.KVH):
            k, v = (torch.where(there[:, None], a[0, pages, h, slots % b.page].double(), 0.0) for a in (b.keys, b.values))
            q = b.q.reshape(b.T, b.H, b.dh)[rows, h * G:(h + 1) * G].double().reshape(n * G, b.dh)
            kt = k.t().contiguous()
            x = (scale * (q @ kt)).masked_fill(~seen, -INF)
            ds = (abs(scale) * (b.dh + 6) * F * (q.abs() @ kt.abs())).masked_fill(~seen, 0.0)
            top = x.amax(1, keepdim=True)
            dead = top == -INF
            top = torch.where(dead, 0.0, top)
            p = torch.exp(x - top)
            e = torch.where(p > 0, ds + ds.amax(1, keepdim=True) + 4 * F * torch.where(seen, x.abs() + top.abs(), 0.0) + 16 * F, 0.0)
            total = torch.where(dead, 1.0, p.sum(1, keepdim=True))
            want, size = p @ v / total, p @ v.abs() / total
            wrong = (p * e) @ v.abs() / total + size * (p * e).sum(1, keepdim=True)
            lost = ((2.0 ** -16 if half else 0.0) + (2 * seen.sum(1, keepdim=True) + 16) * F) * size
            y[rows, h] = want.reshape(n, G, b.dh)
            bounds[rows, h] = (wrong + lost + (M.B16 if half else F) * (want.abs() + wrong + lost) + 1e-38).reshape(n, G, b.dh)
    return y.reshape(b.T, b.H, b.dh), bounds.reshape(b.T, b.H, b.dh)


def _check(b, visible=None, scale=None):
    """b's call against float64, element by element and, for queries and keys of a few units, whose scores leave little, in the mean."""
    y = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=visible, scale=scale).double().reshape(b.T, b.H, b.dh)
    want, bound = _exact(b, visible, scale)
    off = (y - want).abs()
    good = bool((off <= bound).all())
    assert good, (float((off - bound).max()), torch.nonzero(~(off <= bound))[:3].tolist())
    # In the mean: bf16, the result's rounding.  float32: weights 2^-8 of the largest and more, whose exponents span 8, have errors of 1.5 x 2^-24 x 8 (the scale's two
    # roundings), 2^-22 (the exponent's), 2^-22 (the product's, of 64 or 128 terms) and 2^-23 (the exponential's), together below 2^-19, and so has a sum of values of any sign
    mean = float(off.norm() / want.norm().clamp(min=1e-300))
    assert mean <= (M.B16 if b.dtype == torch.bfloat16 else 2.0 ** -19), mean


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
        y = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=visible, scale=scale).double().reshape(b.T, H, dh)
        # The products are exact, so a weight has the roundings of its argument: with the smallest scales, |s| < 6 and a span below 17.4 in base 2, of which the scale's
        # two roundings are 2^-24 and 2^-25, and two roundings of 2^-20, together below 2^-18 of the weight; the exponential's 2^-22 are in it.  Two bf16: 2^-16.  Weights enter
        # twice, above and below; a sum of n of them has n roundings, twice; the result its own
        want, _ = _exact(b, visible, scale)
        half = b.dtype == torch.bfloat16
        n = max(l + c for l, c in zip(lens, nodes))
        wide = float(b.values.abs().max())
        bound = (2 * (2.0 ** -16 if half else 0.0) + 2 * 2.0 ** -18 + (2 * n + 16) * M.F32) * wide + (M.B16 if half else M.F32) * want.abs()
        good = bool(((y - want).abs() <= bound).all())
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
        y = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=visible, scale=scale).double().reshape(b.T, H, dh)
        want, _ = _exact(b, visible, scale)
        # exponents span 24: two roundings of 2^-20 each for a weight and for each of at most 12 rescalings; weights enter twice
        n = max(l + c for l, c in zip(lens, nodes))
        bound = (2 * (2.0 ** -16 if half else 0.0) + 2 * 26 * 2.0 ** -20 + (2 * n + 16) * M.F32) * float(b.values.abs().max()) + (M.B16 if half else M.F32) * want.abs()
        good = bool(((y - want).abs() <= bound).all())
        assert good, float((y - want).abs().max())


# --------------------------------------------------------------------------------------- plans and variants of larger calls
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H", [16, 32, 64])
@pytest.mark.parametrize("page, low", [(8, 480), (8, 600), (16, 900)])
def test_attend_whole_sequences_over_many_pages(dh, H, page, low):
    """More pages than a wave has lanes, in one item: 64, 128 or 256 rows that share their keys; pages that are not there around the 64th and near the end."""
    lens = [low + 61 * i % (1000 - low) for i in range(16)]
    b = Batch(low + H, "bf16", lens, [24 - i % 3 for i in range(16)], H, 8, dh, page)
    assert b.table.shape[1] * page <= 1024                # (whole: 128 pairs of sequence and KV head of up to 1024 slots)
    _check(b)
    _check(b, b.seen())
    for s, gone in enumerate(([63], [64], [61, 62, 63, 64, 65], [0, 63, 64], [66], list(range(58, 64)), [127], [60, 65, 124])):
        for i in gone:
            b.table[s, min(i, b.table.shape[1] - 1)] = -1
    _check(b)
    _check(b, b.seen())


@pytest.mark.parametrize("dh, H, nodes, page", [(128, 8, 24, 8), (64, 8, 24, 16), (128, 4, 20, 8), (64, 20, 24, 8), (128, 16, 20, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_shares_of_many_steps(dtype, dh, H, nodes, page):
    """Contexts of up to 40001 slots whose shares are several steps long, many groups of 64 pages each; some of the pages are not there."""
    b = Batch(H + dh, dtype, [9000, 40001, 23456, 12000], [nodes, nodes - 3, nodes, nodes - 1], H, 2, dh, page)
    _check(b)
    b.table[:, ::37] = -1
    b.table[1, 1000:1130] = b.keys.shape[1]
    _check(b, b.seen())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, H, KVH, dh, most, longest", [(129, 4, 2, 64, 20, 900), (130, 6, 3, 128, 40, 700), (150, 16, 2, 64, 25, 800), (140, 4, 2, 128, 25, 5000),
                                                          (135, 12, 3, 64, 30, 6000), (130, 16, 2, 128, 30, 4000), (200, 8, 8, 128, 1, 3000), (1024, 4, 4, 64, 1, 9000)])
def test_attend_many_sequences_of_several_heads(dtype, n, H, KVH, dh, most, longest):
    """Items that are listed before the launch: blocks of 16 to 256 rows, whole and split, most sequences shorter than a share."""
    g = np.random.default_rng(n)
    lens, nodes = g.integers(0, 300, n), g.integers(max(1, most - 4), most + 1, n)
    lens[[0, n // 2, n - 1]], nodes[3] = longest, 0
    b = Batch(n + dh, dtype, lens.tolist(), nodes.tolist(), H, KVH, dh, 16)
    _check(b)
    _check(b, b.seen())


@pytest.mark.parametrize("n, H, nodes, longest", [(130, 4, 3, 5000), (40, 16, 20, 6000), (150, 16, 20, 900)])
def test_attend_replayed_with_other_lengths(n, H, nodes, longest):
    """A graph of a call whose items are listed before the launch, or counted in it: which sequences are split changes from replay to replay."""
    g = np.random.default_rng(n)
    b = Batch(n, "bf16", [longest] * 3 + [300] * (n - 3), [nodes] * n, H, 2, 64, 16)
    out = torch.zeros_like(b.q)
    most = b.lens.cpu().numpy()

    def run():
        b.cache.attend(0, b.q, b.table, b.lens, b.first, out=out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for turn in range(5):
        b.lens.copy_(_ints((most * g.random(n) ** turn).astype(int).tolist()))
        b.q.copy_(b.normal(b.T, H * 64))
        want = b.cache.attend(0, b.q, b.table, b.lens, b.first)
        torch.cuda.synchronize()
        out.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        _check(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_float32_in_the_mean(dtype):
    """Small batches of both kernels of few rows."""
    for lens, nodes, H, KVH, dh in (([40, 127, 90], [5, 5, 4], 8, 8, 64), ([700, 300], [9, 12], 8, 4, 64), ([1500], [20], 4, 2, 128)):
        b = Batch(sum(lens), dtype, lens, nodes, H, KVH, dh, 16)
        _check(b)
        _check(b, b.seen())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, V, L", [(90, 50257, 300), (700, 50257, 60), (330, 24593, 200)])
def test_logits_in_several_slices(dtype, rows, V, L):
    """Rows past the caches, cut into slices of the vocabulary, one or several rows of a workgroup: tokens, biases and masks on both sides of the slices' borders."""
    g = np.random.default_rng(rows)
    nodes = []
    while sum(nodes) < rows:
        nodes.append(int(min(g.integers(0, 9), rows - sum(nodes))))
    logits, first, kw = _logits_case(V, dtype, len(nodes), nodes, V, L, 40)
    slices = -(-V // 6144)
    slice_ = -(-(-(-V // slices)) // 32) * 32
    edges = np.array([e + d for e in range(0, V + 1, slice_) for d in (-33, -2, -1, 0, 1, 31, 32)])
    edges = np.append(edges, [V - 1, V - 2, V])
    for name in ("tokens", "draft", "bias_ids"):
        a = kw[name]
        kw[name] = np.where(g.random(a.shape) < 0.3, edges[g.integers(0, len(edges), a.shape)], a).astype(np.int32)
    half = dtype == "bf16"
    want = _check_logits(logits, first, kw, half)
    dev = {k: torch.from_numpy(v).to(DEV) for k, v in kw.items()}
    x, f = logits.to(DEV), torch.from_numpy(first).to(DEV)
    assert _ops().adjust_logits(x, f, out=x, **dev) is x and torch.equal(x, want)
    wide = torch.full((rows, V + 9), 3.0, dtype=TYPES[dtype], device=DEV)
    wide[:, 5:V + 5] = logits.to(DEV)
    out = torch.full((rows, V + 6), 3.0, dtype=TYPES[dtype], device=DEV)
    assert torch.equal(_ops().adjust_logits(wide[:, 5:V + 5], f, out=out[:, 3:V + 3], **dev), want)
    assert (out[:, :3] == 3).all() and (out[:, V + 3:] == 3).all()
    _check_logits(logits, first, {k: kw[k] if k in ("draft", "visible", "frequency", "mask", "mask_row") else None for k in kw}, half)


# ------------------------------------------------------------------------------------- committed values that are not finite
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh, page", ENDS)
def test_committed_values_that_are_not_finite(dtype, lens, nodes, H, KVH, dh, page):
    """Infinities of one sign give that infinity, of both signs or NaN give NaN, in their columns alone; as they do in nodes."""
    b = Batch(sum(nodes) + dh, dtype, lens, nodes, H, KVH, dh, page)
    vis = b.seen()
    want, bound = _exact(b, vis)
    what = {3: float("inf"), 7: -float("inf"), 20: float("nan"), 41: None}
    hit = {c: torch.zeros(b.T, dtype=torch.bool, device=DEV) for c in what}
    for s, l in enumerate(lens):
        for n, c in enumerate(what):
            at = sorted({0, l // 2, l - 1, (17 * n) % l} if n != 1 else {l - 1})
            for i, slot in enumerate(at):
                p = M.slot_of(b.table.cpu().numpy(), b.keys.shape[1], page, s, slot)
                b.values[0, p[0], :, p[1], c] = what[c] if what[c] is not None else (-1) ** i * float("inf")
            hit[c][int(b.first[s]):int(b.first[s + 1])] = True
        assert l > 1
    got, again = (b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis).double().reshape(b.T, H, dh) for _ in range(2))
    assert torch.equal(again.nan_to_num(9.0), got.nan_to_num(9.0))
    for c in what:
        y = got[hit[c], :, c]
        good = bool(y.isnan().all() if c > 7 else (y == what[c]).all())
        assert good, (c, y.isnan().float().mean(), (y == float("inf")).float().mean())
    rest = [c for c in range(dh) if c not in what]
    good = bool(((got - want).abs() <= bound)[..., rest].all())
    assert good


def test_committed_values_in_a_few_of_many_sequences():
    """Sequences without infinities keep their bits."""
    for H, nodes in ((4, 1), (16, 6), (16, 20)):
        b = Batch(H + nodes, "bf16", [37 * i % 900 + 2 for i in range(40)], [nodes] * 40, H, 2, 64, 16)
        want = b.cache.attend(0, b.q, b.table, b.lens, b.first)
        rows = torch.zeros(b.T, dtype=torch.bool, device=DEV)
        for s in (0, 7, 39):
            p = M.slot_of(b.table.cpu().numpy(), b.keys.shape[1], 16, s, 1)
            b.values[0, p[0], :, p[1]] = float("inf")
            rows[nodes * s:nodes * (s + 1)] = True
        got = b.cache.attend(0, b.q, b.table, b.lens, b.first)
        assert torch.equal(got[~rows], want[~rows]) and (got[rows] == float("inf")).all()
