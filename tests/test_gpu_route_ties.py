"""Routing where scores of different logits are equal in 64 bits: the lowest index, whatever kernel takes the row and whatever lies beside it."""
import numpy as np
import pytest
import torch
from test_gpu_operators import DEV, _check_route, _ops, _rng

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [12, 40, 200])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_scores_that_meet_next_to_zero(E, score, renormalize):
    """Logits next to zero differ while their scores in 64 bits do not: the lowest index, from either kernel and beside any row."""
    g = _rng(21, E)
    rows = np.full((6, E), -1.0, np.float32)
    rows[:, :4] = [[1e-17, 2e-17, 0.0, -1e-17], [0.0, 1e-20, -0.0, 1e-38], [-1e-18, 1e-18, 3e-18, 0.0], [1e-45, 0.0, 1e-30, 2e-30],
                   [2.0 ** -60, 2.0 ** -59, -2.0 ** -58, 2.0 ** -61], [0.5, 1e-19, 2e-19, 3e-19]]
    rows[:, 4:7] = rows[:, 1:4]
    alone = rows.copy()
    beside = np.concatenate([rows, (g.standard_normal((11, E)) * 2).astype(np.float32)])
    beside[7, 3] = 20.0                                   # (above 16: this row compares scores by itself)
    for kw in (dict(), dict(bias=np.zeros(E, np.float32))):
        for v in (alone, beside, beside[::-1].copy(), np.ascontiguousarray(beside[[0, 7, 3, 8]])):
            _check_route(v, 5, score=score, renormalize=renormalize, **kw)


@pytest.mark.parametrize("E", [16, 64, 250])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_both_kernels_take_the_same_experts(E, score):
    """A bias of zeros and rows of every magnitude: the same ids from the kernel that compares logits and from the one that compares scores."""
    g = _rng(22, E)
    logits = (g.standard_normal((500, E)) * 10.0 ** g.uniform(-20, 2, (500, 1))).astype(np.float32)
    t = torch.from_numpy(logits).to(DEV)
    a = _ops().route(t, 8, score=score)
    b = _ops().route(t, 8, score=score, bias=torch.zeros(E, device=DEV))
    assert torch.equal(a[0], b[0])
    assert ((a[1] - b[1]).abs() <= 2.0 ** -23 * b[1]).all()
    c = _ops().route(t[::7].contiguous(), 8, score=score)
    assert torch.equal(a[0][::7], c[0]) and torch.equal(a[1][::7], c[1])
