"""Routing, the experts' products and the norms around a block against their definitions in float64."""
import numpy as np
import pytest
import torch
import operator_math as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ops():
    from paper_2502_04557_amd import operators
    return operators


def _rng(*key):
    return np.random.default_rng([abs(hash(str(k))) % 1000 if not isinstance(k, int) else k for k in key])


# ------------------------------------------------------------------------------------------------------------------ route
def _check_route(logits, k, **kw):
    bias = kw.pop("bias", None)
    ids, w = _ops().route(logits if isinstance(logits, torch.Tensor) else torch.from_numpy(logits).to(DEV), k,
                          bias=None if bias is None else torch.from_numpy(bias).to(DEV), **kw)
    host = logits.cpu().numpy() if isinstance(logits, torch.Tensor) else logits
    rid, rw = M.route(host, k, bias=bias, **kw)
    assert np.array_equal(ids.cpu().numpy(), rid)
    w = w.cpu().numpy().astype(np.float64)
    assert (np.abs(w - rw) <= M.F32 * rw + 1e-13 * rw + 2.0 ** -149).all()        # float64 inside, rounded once


@pytest.mark.parametrize("T, E, k", [(1, 1, 1), (1, 8, 2), (3, 7, 7), (5, 60, 6), (64, 64, 8), (65, 65, 1), (9, 128, 48), (33, 130, 5),
                                     (17, 256, 8), (4, 257, 3), (6, 1000, 10), (2, 1024, 48), (1500, 16, 4)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_plain(T, E, k, score):
    g = _rng(1, T, E, k)
    logits = (g.standard_normal((T, E)) * 2).astype(np.float32)
    _check_route(logits, k, score=score)
    _check_route(logits, k, score=score, renormalize=False, scale=2.5, n_shared=2, bias=(g.standard_normal(E) * 0.1).astype(np.float32))


@pytest.mark.parametrize("E, G, top, k", [(8, 2, 1, 2), (12, 3, 2, 5), (64, 64, 7, 7), (60, 4, 3, 8), (256, 8, 4, 8), (1024, 16, 2, 6),
                                          (130, 10, 10, 4), (96, 32, 5, 3)])
@pytest.mark.parametrize("how", ["max", "sum2"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_groups(E, G, top, k, how, score):
    g = _rng(2, E, G, top)
    logits = g.standard_normal((37, E)).astype(np.float32)
    logits[g.random((37, E)) < 0.2] = -np.inf
    logits[5] = -np.inf
    logits[6, : E // 2] = -np.inf
    _check_route(logits, k, score=score, n_group=G, top_group=top, group_score=how)
    _check_route(logits, k, score=score, n_group=G, top_group=top, group_score=how, bias=(g.standard_normal(E) * 0.2 - 0.3).astype(np.float32))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_masks_ties_and_extremes(score):
    g = _rng(3)
    E = 40
    logits = g.integers(-3, 4, (64, E)).astype(np.float32)           # many equal ones: the lowest index
    logits[0] = -np.inf                                              # nobody left
    logits[1, 1:] = -np.inf
    logits[2, ::2] = np.nan
    logits[3, 7] = np.inf
    logits[4, [3, 9]] = np.inf
    logits[5] = np.finfo(np.float32).min                             # a mask of the lowest value leaves equal ones
    logits[6, 1:] = np.finfo(np.float32).min
    logits[7] = 200.0 * g.standard_normal(E)
    logits[8] = 0.0
    logits[9] = -0.0
    logits[9, 5] = 0.0
    for kw in (dict(), dict(renormalize=False, n_shared=1), dict(bias=np.where(np.arange(E) % 3 == 0, -np.inf, 0.5).astype(np.float32))):
        _check_route(logits, 6, score=score, **kw)


def test_route_rows_apart_and_no_rows():
    g = _rng(4)
    wide = torch.from_numpy(g.standard_normal((20, 77)).astype(np.float32)).to(DEV)
    _check_route(wide[:, 5:69], 4)
    _check_route(wide[::3, 1:9], 2)
    ids, w = _ops().route(wide[:0, :8], 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)


# ---------------------------------------------------------------------------------------------------------------- experts
def _weights(E, d, ff, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dt=dtype):
        return torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, std, generator=g)

    return normal(E, ff, d, std=d ** -0.5), normal(E, ff, d, std=d ** -0.5), normal(E, d, ff, std=ff ** -0.5), normal, g


def _check_experts(y, x, ids, w, mats):
    ref, bound = M.experts(x.double(), ids.long(), w.double(), *(m.double() for m in mats), half=x.dtype == torch.bfloat16)
    off = (y.double() - ref).abs()
    assert torch.isfinite(y).all()
    bad = off > bound
    assert not bad.any(), (int(bad.sum()), float((off / bound).max()), bad.nonzero()[:4].tolist())


BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T, E, k, d, ff", [
    (1, 1, 1, 8, 8), (1, 8, 2, 256, 704), (2, 4, 4, 40, 24), (7, 8, 2, 512, 1344), (16, 64, 8, 128, 72), (16, 3, 1, 264, 520),
    (17, 8, 2, 256, 704), (31, 5, 3, 200, 136), (64, 16, 4, 320, 200), (100, 8, 2, 768, 1088), (257, 9, 2, 136, 264), (400, 4, 1, 256, 256),
    (900, 6, 3, 328, 712), (2100, 4, 2, 256, 384), (1500, 5, 4, 520, 264)])
def test_experts(T, E, k, d, ff, dtype):
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, T * 1000 + E)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    _check_experts(_ops().Experts(wg, wu, w2)(x, ids, w), x, ids, w, (wg, wu, w2))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [1, 13, 60, 300, 1200])
def test_experts_uneven_dropped_and_named_twice(T, dtype):
    E, k, d, ff = 12, 4, 264, 200
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, T)
    x = normal(T, d)
    ids = torch.randint(-1, 3, (T, k), generator=g, device=DEV, dtype=torch.int32)      # three busy experts, the same one twice, none
    ids[T // 2] = -1
    ids[T // 3, 0] = 11
    ids[0, k - 1] = 2 ** 30                                                             # no expert of this device
    ids[T - 1, 0] = -2 ** 31
    w = torch.rand(T, k, generator=g, device=DEV)
    # what stands beside an id without an expert is not read into the sum
    w = torch.where((ids < 0) | (ids >= E), torch.full_like(w, float("nan")), w)
    y = _ops().Experts(wg, wu, w2)(x, ids, w)
    some = (ids >= 0) & (ids < E)
    _check_experts(y, x, torch.where(some, ids, -1), torch.where(some, w, 0.0), (wg, wu, w2))
    if T > 2:
        assert (y[T // 2] == 0).all()
    none = _ops().Experts(wg, wu, w2)(x, torch.full_like(ids, -1), w)
    assert (none == 0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [5, 40, 700])
def test_experts_rows_do_not_meet(T, dtype):
    """Infinities and NaN stay in their row, whatever lies beside it; rows of x and y lie apart, and what lies between is left as it was."""
    E, k, d, ff = 4, 2, 136, 264
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, T + 7)
    wide = normal(T + 3, d + 24)
    x = wide[:T, 8:8 + d]
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    experts = _ops().Experts(wg, wu, w2)
    clean = experts(x, ids, w)
    wide[1, 9] = float("inf")
    wide[T - 1, 20] = float("nan")
    wide[:, :8] = float("nan")
    wide[T:] = float("nan")
    room = torch.full((T + 2, d + 16), 7.0, dtype=dtype, device=DEV)
    out = experts(x, ids, w, out=room[1:T + 1, 8:8 + d])
    assert out.data_ptr() == room[1:, 8:].data_ptr()
    assert not torch.isfinite(out[1]).all() and not torch.isfinite(out[T - 1]).any()
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[1] = keep[T - 1] = False
    assert torch.equal(out[keep], clean[keep])
    room[1:T + 1, 8:8 + d] = 7.0
    assert (room == 7.0).all()


@pytest.mark.parametrize("d, ff, T", [(1032, 5480, 1200), (264, 200, 1200)])
def test_experts_short_blocks(d, ff, T):
    """One row, and 20 and 100 rows, of an expert among row blocks of 256 and of 128."""
    wg, wu, w2, normal, g = _weights(6, d, ff, BF, T)
    x = normal(T, d)
    ids = torch.randint(0, 3, (T, 4), generator=g, device=DEV, dtype=torch.int32)
    ids[7, 0] = 3
    ids[100:120, 1] = 4
    ids[200:300, 2] = 5
    w = torch.rand(T, 4, generator=g, device=DEV)
    experts = _ops().Experts(wg, wu, w2)
    _poison()
    _check_experts(experts(x, ids, w), x, ids, w, (wg, wu, w2))


@pytest.mark.parametrize("T", [1, 16, 17, 600])
@pytest.mark.parametrize("scale", [1e-6, 1e4])
def test_experts_small_and_large_weights(T, scale):
    """A row's weights scale its result and nothing else."""
    wg, wu, w2, normal, g = _weights(5, 128, 96, BF, T)
    x = normal(T, 128)
    ids, w = _ops().route(normal(T, 5, dt=FP), 2, scale=scale)
    _check_experts(_ops().Experts(wg, wu, w2)(x, ids, w), x, ids, w, (wg, wu, w2))


def _poison():
    """Memory that later allocations take holds NaN."""
    t = torch.full((1 << 28,), float("nan"), device=DEV)
    del t


@pytest.mark.parametrize("T, E, k, d, ff", [(3, 20, 6, 72, 40), (2100, 4, 2, 1032, 5480), (700, 4, 2, 520, 1352), (90, 4, 1, 264, 200)])
def test_experts_odd_columns_in_every_tile(T, E, k, d, ff):
    """Columns behind d and d_ff in the last k tile, on a workspace full of NaN: few rows, 256 x 256, 128 x 128, 64 x 128."""
    wg, wu, w2, normal, g = _weights(E, d, ff, BF, T)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    experts = _ops().Experts(wg, wu, w2)
    _poison()
    _check_experts(experts(x, ids, w), x, ids, w, (wg, wu, w2))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [4, 16, 50, 600])
def test_experts_broken_expert(T, dtype):
    """What an expert's weights hold reaches the rows that name it, and no other."""
    E, k, d, ff = 6, 2, 128, 96
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, T)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    clean = _ops().Experts(wg, wu, w2)(x, ids, w)
    w2[2, 5], wu[3, 7] = float("inf"), float("nan")
    y = _ops().Experts(wg, wu, w2)(x, ids, w)
    touched = ((ids == 2) | (ids == 3)).any(1)
    assert torch.equal(y[~touched], clean[~touched])
    assert not torch.isfinite(y[touched]).all(1).any()


@pytest.mark.parametrize("T", [1, 30, 500])
def test_experts_again_and_beside_other_rows(T):
    """The same rows give the same bits on every run, and in another order of the batch."""
    E, k, d, ff = 8, 2, 256, 320
    wg, wu, w2, normal, g = _weights(E, d, ff, BF, 5)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    experts = _ops().Experts(wg, wu, w2)
    y = experts(x, ids, w)
    assert torch.equal(experts(x, ids, w), y)
    order = torch.randperm(T, generator=g, device=DEV)
    assert torch.equal(experts(x[order].contiguous(), ids[order].contiguous(), w[order].contiguous()), y[order])


# ----------------------------------------------------------------------------------------------------------------- block norm
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T, d", [(1, 1), (3, 2), (2, 7), (5, 64), (4, 250), (3, 768), (9, 1000), (2, 1601), (6, 2048), (3, 4096), (2, 4097),
                                  (2, 8192), (1, 12345), (2, 16384), (300, 512)])
@pytest.mark.parametrize("post, gate, scale", [(True, "column", 0.5), (False, None, 1.0), (True, "row", 0.22), (False, "both", -1.5)])
def test_block_norm(T, d, kind, dtype, post, gate, scale):
    g = _rng(6, T, d)

    def f(*shape, mean=0.0, std=1.0):
        return (mean + std * g.standard_normal(shape)).astype(np.float32)

    h, y = f(T, d, mean=0.3, std=3), torch.from_numpy(f(T, d, mean=-0.2)).to(dtype)
    gain, offset = f(d, mean=1, std=0.1), f(d) if kind == "layer" else None
    pg, pb = (f(d, mean=1, std=0.1), f(d, std=0.1) if kind == "layer" else None) if post else (None, None)
    gt = {None: None, "column": f(1, d), "row": f(T, 1), "both": f(T, d)}[gate]
    dev = [None if a is None else torch.from_numpy(a).to(DEV) for a in (h, gain, offset, pg, pb, gt)]
    hn, out = _ops().block_norm(dev[0], y.to(DEV), dev[1], offset=dev[2], post_gain=dev[3], post_offset=dev[4], gate=dev[5], scale=scale, kind=kind)
    assert torch.equal(dev[0].cpu(), torch.from_numpy(h)) and out.dtype == dtype
    wide = [None if a is None else a.astype(np.float64) for a in (h, gain, offset, pg, pb, gt)]
    rh, bh, ro, bo = M.block_norm(wide[0], y.double().numpy(), wide[1], wide[2], wide[3], wide[4], wide[5], float(np.float32(scale)),
                                  float(np.float32(1e-5)), kind, dtype == BF)
    assert (np.abs(hn.cpu().double().numpy() - rh) <= bh).all()
    assert (np.abs(out.cpu().double().numpy() - ro) <= bo).all()


@pytest.mark.parametrize("d", [40, 129, 4096])
def test_block_norm_in_place_rows_apart(d):
    g = _rng(7, d)
    T = 11
    wide = torch.from_numpy(g.standard_normal((T + 2, d + 5)).astype(np.float32)).to(DEV)
    ywide = torch.from_numpy(g.standard_normal((T, d + 3)).astype(np.float32)).to(DEV).to(BF)
    gain = torch.from_numpy(g.standard_normal(d).astype(np.float32)).to(DEV)
    h, y = wide[1:T + 1, 2:2 + d], ywide[:, 1:1 + d]
    before = wide.clone()
    hn, out = _ops().block_norm(h.contiguous(), y.contiguous(), gain, post_gain=gain)
    got, out2 = _ops().block_norm(h, y, gain, post_gain=gain, h_out=h)
    assert got.data_ptr() == h.data_ptr()
    rh, bh, ro, bo = M.block_norm(before[1:T + 1, 2:2 + d].cpu().double().numpy(), y.cpu().double().numpy(), gain.cpu().double().numpy(),
                                  post_gain=gain.cpu().double().numpy(), eps=float(np.float32(1e-5)), half=True)
    for a, o in ((hn, out), (h, out2)):
        assert (np.abs(a.cpu().double().numpy() - rh) <= bh).all() and (np.abs(o.cpu().double().numpy() - ro) <= bo).all()
    before[1:T + 1, 2:2 + d] = wide[1:T + 1, 2:2 + d]
    assert torch.equal(before, wide)


def test_block_norm_rows_do_not_meet():
    T, d = 6, 512
    g = _rng(8)
    h = torch.from_numpy(g.standard_normal((T, d)).astype(np.float32)).to(DEV)
    y = torch.from_numpy(g.standard_normal((T, d)).astype(np.float32)).to(DEV)
    gain = torch.ones(d, device=DEV)
    hn, out = _ops().block_norm(h, y, gain, post_gain=gain)
    y[2, 5], h[4, 7] = float("nan"), float("inf")
    y[5], h[5] = 0.0, 0.0
    hn2, out2 = _ops().block_norm(h, y, gain, post_gain=gain)
    assert torch.isnan(out2[2]).all() and torch.isnan(hn2[2]).all() and torch.isinf(hn2[4, 7])
    assert (out2[5] == 0).all()
    for r in (0, 1, 3):
        assert torch.equal(hn[r], hn2[r]) and torch.equal(out[r], out2[r])


# ------------------------------------------------------------------------------------------------------------- limits, refusals
@pytest.mark.parametrize("T, E, k, d, ff", [(16, 1024, 8, 64, 24), (40, 600, 48, 64, 40), (3, 70, 60, 64, 16), (1, 1024, 64, 72, 8),
                                            (16, 64, 64, 64, 32), (17, 1024, 1, 64, 64), (2000, 1024, 4, 64, 64)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_experts_many_experts(T, E, k, d, ff, dtype):
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, E + k)
    x = normal(T, d)
    ids = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].to(torch.int32).contiguous()
    w = torch.rand(T, k, generator=g, device=DEV)
    _check_experts(_ops().Experts(wg, wu, w2)(x, ids, w), x, ids, w, (wg, wu, w2))


@pytest.mark.parametrize("T", [3, 40])
def test_experts_weights_beyond_32_bits(T):
    E, d, ff = 40, 4096, 14336                           # 4.7 GB a matrix
    wg, wu, w2, normal, g = _weights(E, d, ff, BF, T)
    x = normal(T, d)
    ids = torch.full((T, 2), E - 1, dtype=torch.int32, device=DEV)
    ids[:, 1] = 36
    w = torch.rand(T, 2, generator=g, device=DEV)
    y = _ops().Experts(wg, wu, w2)(x, ids, w)
    _check_experts(y, x, torch.where(ids == 36, 0, 1), w, tuple(m[[36, E - 1]] for m in (wg, wu, w2)))


def test_rows_beyond_32_bits():
    T, d = 530000, 4096                                  # 2.2e9 elements
    h = torch.zeros(T, d, device=DEV)
    y = torch.zeros(T, d, dtype=BF, device=DEV)
    g = _rng(9)
    last = g.standard_normal((5, d)).astype(np.float32)
    h[-5:] = torch.from_numpy(last).to(DEV)
    y[-5:] = torch.from_numpy(last[::-1].copy()).to(DEV).to(BF)
    gain = torch.ones(d, device=DEV)
    hn, out = _ops().block_norm(h, y, gain, post_gain=gain)
    rh, bh, ro, bo = M.block_norm(last.astype(np.float64), y[-5:].cpu().double().numpy(), np.ones(d), post_gain=np.ones(d),
                                  eps=float(np.float32(1e-5)), half=True)
    assert (np.abs(hn[-5:].cpu().double().numpy() - rh) <= bh).all() and (np.abs(out[-5:].cpu().double().numpy() - ro) <= bo).all()
    assert (hn[:-5:1000] == 0).all() and (out[:-5:1000] == 0).all()
    del h, y, hn, out
    T, E = 1 << 23, 264                                  # the most rows
    logits = torch.zeros(T, E, device=DEV)
    logits[-3:] = torch.from_numpy(g.standard_normal((3, E)).astype(np.float32)).to(DEV)
    for bias in (None, np.zeros(E, np.float32)):
        ids, w = _ops().route(logits, 3, bias=None if bias is None else torch.from_numpy(bias).to(DEV))
        rid, _ = M.route(logits[-3:].cpu().numpy(), 3, bias=bias)
        assert np.array_equal(ids[-3:].cpu().numpy(), rid) and (ids[:-3:4096].cpu() == torch.arange(3)).all()


def test_wrong_tensors_are_refused():
    from paper_2502_04557_amd.binding import SprinterError
    ops = _ops()
    f = lambda *s, dt=FP: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
    for bad in (f(4, 8, dt=BF), f(8), f(8, 4).t(), f(4, 8).requires_grad_()):
        with pytest.raises(ValueError):
            ops.route(bad, 2)
    with pytest.raises(ValueError):
        ops.route(f(4, 8), 2, bias=f(7))
    with pytest.raises(ValueError):
        ops.route(f(4, 8), 2, bias=torch.zeros(8))
    with pytest.raises(ValueError):
        ops.route(f(4, 8), 2, score="linear")
    with pytest.raises(SprinterError, match="top_k"):
        ops.route(f(4, 8), 9)
    with torch.no_grad():
        ops.route(f(4, 8).requires_grad_(), 2)
    e = ops.Experts(f(4, 16, 8, dt=BF), f(4, 16, 8, dt=BF), f(4, 8, 16, dt=BF))
    ids, w = torch.zeros(3, 2, dtype=torch.int32, device=DEV), f(3, 2)
    with pytest.raises(ValueError):
        ops.Experts(f(4, 16, 8, dt=BF), f(4, 16, 8, dt=BF), f(4, 16, 8, dt=BF))
    for x, i, ww in ((f(3, 8), ids, w), (f(3, 16, dt=BF), ids, w), (f(3, 8, dt=BF), ids.long(), w), (f(3, 8, dt=BF), ids[:2], w),
                     (f(3, 8, dt=BF), ids, w.to(BF)), (f(3, 8, dt=BF), ids.t().contiguous().t(), w), (f(3, 8, dt=BF), None, w)):
        with pytest.raises(ValueError):
            e(x, i, ww)
    with pytest.raises(SprinterError, match="16-byte"):
        e(f(3, 12, dt=BF)[:, 2:10], ids, w)
    with pytest.raises(SprinterError, match="columns"):
        e(f(1, 8, dt=BF).expand(3, 8), ids, w)
    assert e(f(0, 8, dt=BF), ids[:0], w[:0]).shape == (0, 8)
    h, y, g = f(3, 8), f(3, 8, dt=BF), f(8)
    for kw in (dict(gain=f(7)), dict(gain=g, gate=f(2, 8)), dict(gain=g, gate=f(8, dt=BF)), dict(gain=g, kind="batch"), dict(gain=g, h_out=f(3, 7)),
               dict(gain=g, offset=f(8, dt=BF)), dict(gain=g.requires_grad_())):
        with pytest.raises(ValueError):
            ops.block_norm(h, y, **kw)
    with pytest.raises(ValueError):
        ops.block_norm(h, y.to(torch.float16), g)
    with pytest.raises(SprinterError, match="post_offset"):
        ops.block_norm(h, y, f(8), post_offset=f(8))
    assert ops.block_norm(h[:0], y[:0], f(8))[1].shape == (0, 8)


# ------------------------------------------------------------------------------------------------------------- run together
def _block(E=8, d=256, ff=320, k=2, shared=1, seed=3, dtype=BF):
    wg, wu, w2, normal, g = _weights(E + shared, d, ff, dtype, seed)
    router = normal(E, d, std=d ** -0.5, dt=FP)
    gain = 1 + 0.1 * normal(d, dt=FP)
    return dict(experts=_ops().Experts(wg, wu, w2), mats=(wg, wu, w2), router=router, gain=gain, post=1 + 0.1 * normal(d, dt=FP),
                gate=normal(1, d, dt=FP), k=k, shared=shared, normal=normal, d=d)


def _run_block(b, x, h):
    logits = x.float() @ b["router"].t()
    ids, w = _ops().route(logits, b["k"], score="sigmoid", scale=1.5, n_shared=b["shared"])
    y = b["experts"](x, ids, w)
    hn, out = _ops().block_norm(h, y, b["gain"], post_gain=b["post"], gate=b["gate"], scale=0.5)
    return logits, ids, w, y, hn, out


@pytest.mark.parametrize("T", [1, 16, 50, 600])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_block(T, dtype):
    b = _block(dtype=dtype)
    x, h = b["normal"](T, b["d"]), b["normal"](T, b["d"], dt=FP)
    logits, ids, w, y, hn, out = _run_block(b, x, h)
    rid, rw = M.route(logits.cpu().numpy(), b["k"], score="sigmoid", scale=1.5, n_shared=b["shared"])
    assert np.array_equal(ids.cpu().numpy(), rid)
    _check_experts(y, x, ids, w, b["mats"])
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    rh, bh, ro, bo = M.block_norm(f64(h), f64(y), f64(b["gain"]), post_gain=f64(b["post"]), gate=f64(b["gate"]), scale=0.5,
                                  eps=float(np.float32(1e-5)), half=dtype == BF)
    assert (np.abs(f64(hn) - rh) <= bh).all() and (np.abs(f64(out) - ro) <= bo).all()


@pytest.mark.parametrize("T", [1, 24, 700])
def test_captured_and_replayed(T):
    """The three operators in one graph, replayed on new inputs, with eager work between the replays; and a second graph of the same
    experts whose replays alternate with the first one's."""
    b = _block()
    xs = [b["normal"](T, b["d"]) for _ in range(2)]
    hs = [b["normal"](T, b["d"], dt=FP) for _ in range(2)]
    ids_w = [None, None]
    graphs, outs = [], []
    for i in range(2):
        logits = xs[i].float() @ b["router"].t()

        def run(i=i, logits=logits):
            ids, w = _ops().route(logits, b["k"], n_shared=b["shared"])
            y = b["experts"](xs[i], ids, w)
            return (ids, w, y) + _ops().block_norm(hs[i], y, b["gain"], post_gain=b["post"])

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run())
        graphs.append((g, run))
    for n in range(4):
        for i in range(2):
            xs[i].copy_(b["normal"](T, b["d"]))
            graphs[i][0].replay()
            torch.cuda.synchronize()
            want = graphs[i][1]()
            for a, e in zip(outs[i], want):
                assert torch.equal(a, e)


def test_two_streams_at_once():
    b = _block()
    T = 300
    xs = [b["normal"](T, b["d"]) for _ in range(2)]
    ids, w = _ops().route(b["normal"](T, 8, dt=FP), 2)
    want = [b["experts"](x, ids, w) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(b["experts"](xs[i], ids, w))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])
