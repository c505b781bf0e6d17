"""The operators once more: what rounding alone may leave of the experts, tile by tile; replays whose routing changes; rows that a
workgroup of the norm takes one after the other; the widest rows of any alignment."""
import numpy as np
import pytest
import torch
import operator_checks as K
import operator_math as M
from test_gpu_operators import BF, DEV, FP, _ops, _poison, _rng, _weights
from test_operator_checks import SHAPES

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------------------ block norm
def _norm_case(T, d, kind, dtype, post, gate, apart, g):
    def f(*shape, mean=0.0, std=1.0):
        return (mean + std * g.standard_normal(shape)).astype(np.float32)

    layer = kind == "layer"
    v = dict(h=f(T, d, mean=0.3, std=3), gain=f(d, mean=1, std=0.1), offset=f(d) if layer else None,
             post_gain=f(d, mean=1, std=0.1) if post else None, post_offset=f(d, std=0.1) if post and layer else None,
             gate={None: None, "column": f(1, d), "row": f(T, 1), "both": f(T, d)}[gate])
    y = torch.from_numpy(f(T, d, mean=-0.2)).to(dtype)
    dev = {k: None if a is None else torch.from_numpy(a).to(DEV) for k, a in v.items()}
    h = dev.pop("h")
    if apart:
        wide = torch.empty(T, d + apart, device=DEV)
        wide[:, :d] = h
        h = wide[:, :d]
    hn, out = _ops().block_norm(h, y.to(DEV), scale=0.5, kind=kind, **dev)
    v = {k: None if a is None else a.astype(np.float64) for k, a in v.items()}
    rh, bh, ro, bo = M.block_norm(v.pop("h"), y.double().numpy(), v.pop("gain"), v.pop("offset"), scale=0.5, eps=float(np.float32(1e-5)), kind=kind,
                                  half=dtype == BF, **v)
    assert (np.abs(hn.cpu().double().numpy() - rh) <= bh).all()
    assert (np.abs(out.cpu().double().numpy() - ro) <= bo).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [520, 2056])
@pytest.mark.parametrize("post, gate", [(True, "both"), (True, "row"), (False, "column"), (True, None)])
def test_block_norm_rows_one_after_the_other(d, kind, dtype, post, gate):
    """More rows than there are workgroups: two, three and four to a workgroup, every one of them of live data."""
    _norm_case(6500, d, kind, dtype, post, gate, 0, _rng(23, d))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d, apart", [(16381, 0), (16382, 1), (16383, 0), (16384, 1), (16384, 3)])
def test_block_norm_widest_rows_of_any_alignment(d, apart, kind, dtype):
    """The row in LDS and the sums beside it are more than 64 KiB."""
    _norm_case(3, d, kind, dtype, True, "column", apart, _rng(24, d))


# --------------------------------------------------------------------------------------------------------------------------- experts
def _check_tiles(y, x, ids, w, mats=None, one=None):
    half = x.dtype == BF
    ref, expected = K.experts(x.double(), ids.long(), w.double(), *(m.double() for m in mats or (x, x, x)), half, one)
    worst = K.worst_tile(y, ref, expected, half)
    assert worst <= 1.0, worst
    return worst


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T, E, k, d, ff", SHAPES + [(2100, 4, 2, 1032, 5480), (400, 4, 1, 256, 256), (512, 16, 4, 1024, 2048)])
def test_experts_tile_by_tile(T, E, k, d, ff, dtype):
    wg, wu, w2, normal, g = _weights(E, d, ff, dtype, T * 1000 + E)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), k)
    experts = _ops().Experts(wg, wu, w2)
    _poison()
    print("share of the bound", T, E, k, d, ff, _check_tiles(experts(x, ids, w), x, ids, w, (wg, wu, w2)), flush=True)


@pytest.mark.parametrize("T", [1, 3, 16, 17, 61, 600])
def test_experts_of_wide_models_tile_by_tile(T):
    E, d, ff = 6, 4096, 14336
    wg, wu, w2, normal, g = _weights(E, d, ff, BF, T)
    x = normal(T, d)
    ids, w = _ops().route(normal(T, E, dt=FP), 2)
    y = _ops().Experts(wg, wu, w2)(x, ids, w)
    print("share of the bound", T, _check_tiles(y, x, ids, w, one=lambda e: (wg[e].double(), wu[e].double(), w2[e].double())), flush=True)


# --------------------------------------------------------------------------------------------------------- replays of other routing
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [1, 16, 24, 700])
def test_replays_whose_routing_changes(T, dtype):
    """Two graphs of the three operators whose replays alternate; before each the rows, the residual rows and the logits change: rows
    evenly spread, all of them on two experts, an expert that nobody takes, rows without any expert.  So the experts named, their
    slots, the row blocks and how many there are differ from replay to replay under one captured grid."""
    E, d, ff, k = 10, 264, 328, 2
    wg, wu, w2, normal, g = _weights(E + 1, d, ff, dtype, T)
    experts = _ops().Experts(wg, wu, w2)
    gain, post, gate = 1 + 0.1 * normal(d, dt=FP), 1 + 0.1 * normal(d, dt=FP), normal(T, d, dt=FP)

    def skews():
        plain = normal(T, E, dt=FP)
        two, none, off = plain.clone(), plain.clone(), plain.clone()
        two[:, [3, 7]] += 60.0
        none[:, 5] = -float("inf")
        off[::3] = -float("inf")
        return [plain, two, none, off, normal(T, E, dt=FP)]

    sides = []
    for i in range(2):
        s = dict(x=normal(T, d), h=normal(T, d, dt=FP), logits=normal(T, E, dt=FP))

        def run(s=s, shared=i):
            ids, w = _ops().route(s["logits"], k, n_shared=shared, score=("softmax", "sigmoid")[shared])
            y = experts(s["x"], ids, w)
            return (ids, w, y) + _ops().block_norm(s["h"], y, gain, post_gain=post, gate=gate, scale=0.5)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s["out"] = run()
        sides.append((s, run, graph))
    seen = [[], []]
    for logits in skews() + skews()[::-1]:
        for i, (s, run, graph) in enumerate(sides):
            s["x"].copy_(normal(T, d))
            s["h"].copy_(normal(T, d, dt=FP))
            s["logits"].copy_(logits.roll(i, 0))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in s["out"]]
            want = run()
            for a, e in zip(got, want):
                assert torch.equal(a, e)
            ref, expected = K.experts(s["x"].double(), got[0].long(), got[1].double(), wg.double(), wu.double(), w2.double(), dtype == BF)
            assert K.worst_tile(got[2], ref, expected, dtype == BF) <= 1.0
            seen[i].append(got[0].cpu().numpy().tobytes())
    assert all(len(set(ids)) >= 8 for ids in seen) or T == 1 and all(len(set(ids)) >= 4 for ids in seen)
