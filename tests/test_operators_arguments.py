"""What the torch entry points of the operators make of their arguments before the library sees them, on the CPU."""
import ctypes as C
import pytest
import torch
from test_abi_cpu import lib  # noqa: F401
from paper_2502_04557_amd import operators as ops

ROUTE = dict(n_expert=8, top_k=2, score="softmax", n_group=1, top_group=1, group_score="max", renormalize=True, n_shared=0, scale=1.0)


# ------------------------------------------------------------------------------------- numbers beyond the library's 32 bits
@pytest.mark.parametrize("change", [dict(n_shared=-2 ** 32), dict(n_shared=2 ** 32), dict(top_k=2 ** 32 + 2), dict(top_k=2 - 2 ** 32), dict(n_group=2 ** 32 + 1),
                                    dict(top_group=2 ** 31), dict(n_expert=2 ** 32 + 8), dict(top_k=-2 ** 31 - 1)])
def test_a_number_beyond_32_bits_is_refused(change):
    """Cut off, n_shared = -2^32 would be 0 in the library and leave the outputs, made for top_k - 2^32 columns, without room."""
    with pytest.raises(ValueError, match="32 bits"):
        ops._route_cfg(*{**ROUTE, **change}.values())


def test_shapes_beyond_32_bits_are_refused(lib):  # noqa: F811
    meta = torch.device("meta")
    for rows in (2 ** 31, 2 ** 32 + 5):
        with pytest.raises(ValueError, match="32 bits"):
            ops._rows("x", torch.empty(rows, 8, device=meta), meta, torch.float32, None, 8)
    ops._rows("x", torch.empty(2 ** 31 - 1, 8, device=meta), meta, torch.float32, None, 8)
    with pytest.raises(ValueError, match="32 bits"):
        ops._norm_cfg(torch.float32, "rms", 2 ** 32 + 64, 1e-5, 1.0)
    e = ops.Experts.__new__(ops.Experts)
    cfg = ops.ExpertsCfgC(1, 8, 64, 128)
    e._ref, e._need = C.byref(cfg), {}
    for rows, k in ((2 ** 32 + 1, 2), (1, 2 ** 32 + 2)):
        with pytest.raises(ValueError, match="32 bits"):
            e._bytes(rows, k)
    assert e._bytes(4, 2)[2] > 0


# ------------------------------------------------------------------------------------------- numbers that can change in place
@pytest.mark.parametrize("change", [dict(scale=torch.tensor(2.5)), dict(scale=torch.nn.Parameter(torch.tensor(2.5))), dict(renormalize=torch.tensor(True)),
                                    dict(top_k=torch.tensor(2)), dict(scale="2.5"), dict(scale=None)])
def test_an_option_of_a_route_is_a_plain_number(change):
    """A tensor is the same key of the kept configurations after its value has changed, so the old value would be used again."""
    with pytest.raises(ValueError):
        ops._route_cfg(*{**ROUTE, **change}.values())


def test_an_option_of_a_norm_is_a_plain_number():
    scale = torch.tensor(0.5)
    for eps, s in ((1e-5, scale), (torch.tensor(1e-5), 1.0)):
        with pytest.raises(ValueError, match="plain number"):
            ops._norm_cfg(torch.float32, "rms", 64, eps, s)
    import numpy as np
    assert ops._norm_cfg(torch.float32, "rms", 64, np.float32(1e-5), float(scale))[0].scale == 0.5
    assert ops._route_cfg(*{**ROUTE, "top_k": np.int64(2), "scale": np.float64(2.5)}.values())[0].scale == 2.5
    assert ops._route_cfg(*{**ROUTE, "renormalize": False}.values())[0].renormalize == 0
