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


# ------------------------------------------------------------------------------------------------------- gradients, versions
CPU = torch.device("cpu")


@pytest.fixture
def no_device(monkeypatch):
    """The entry points up to the library's own call, on tensors of the CPU."""
    calls = []
    monkeypatch.setattr(ops, "_device", lambda t, name: t.device)
    monkeypatch.setattr(ops, "_call", lambda name, *args: calls.append(name))
    return calls


def _experts():
    return ops.Experts(torch.ones(4, 16, 8), torch.ones(4, 16, 8), torch.ones(4, 8, 16))


def test_tangents_are_refused(no_device, lib):  # noqa: F811
    import torch.autograd.forward_ad as fwd
    f = lambda *s: torch.ones(*s)  # noqa: E731
    ids, e = torch.zeros(3, 2, dtype=torch.int32), _experts()
    with fwd.dual_level():
        dual = lambda *s: fwd.make_dual(f(*s), f(*s))  # noqa: E731
        for call in (lambda: ops.route(dual(3, 8), 2), lambda: ops.route(f(3, 8), 2, bias=dual(8)), lambda: e(dual(3, 8), ids, f(3, 2)),
                     lambda: e(f(3, 8), ids, dual(3, 2)), lambda: ops.Experts(dual(4, 16, 8), f(4, 16, 8), f(4, 8, 16)),
                     lambda: ops.block_norm(dual(3, 8), f(3, 8), f(8)), lambda: ops.block_norm(f(3, 8), dual(3, 8), f(8)),
                     lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), gate=dual(8))):
            with pytest.raises(ValueError, match="tangent"):
                call()
        ops.route(f(3, 8), 2)                            # plain tensors pass beside dual ones
        ops.route(fwd.unpack_dual(dual(3, 8)).primal, 2)
    assert no_device == ["sprinter_route"] * 2


def test_a_tensor_written_in_place_is_known_to_autograd(no_device, lib):  # noqa: F811
    """What autograd has saved for a backward pass and is then written by out= or h_out= makes that pass an error, not a wrong gradient."""
    ids, w, e = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, 2), _experts()
    for write in (lambda t: e(torch.ones(3, 8), ids, w, out=t), lambda t: ops.block_norm(t, torch.ones(3, 8), torch.ones(8), h_out=t),
                  lambda t: ops.block_norm(torch.ones(3, 8), torch.ones(3, 8), torch.ones(8), h_out=t)):
        leaf, t = torch.ones(3, 8, requires_grad=True), torch.ones(3, 8)
        loss = (leaf * t).sum()
        assert write(t)[0].shape[-1] == 8 and t._version == 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    assert ops.block_norm(torch.ones(3, 8), torch.ones(3, 8), torch.ones(8))[0]._version == 0


def test_truth_values_of_numpy(no_device, monkeypatch):
    import numpy as np
    seen = []
    monkeypatch.setattr(ops, "_call", lambda name, dev, cfg, *args: seen.append(cfg._obj.renormalize))
    for v in (True, np.True_, 1, False, np.False_, 0):
        ops._route_cfg.cache_clear()                     # (True and np.True_ are one key)
        ops.route(torch.ones(3, 8), 2, renormalize=v)
    assert seen == [1, 1, 1, 0, 0, 0]
    with pytest.raises(ValueError, match="renormalize"):
        ops.route(torch.ones(3, 8), 2, renormalize=torch.tensor(True))


def test_negated_views_are_refused(no_device, lib):  # noqa: F811
    """The imaginary part of a conjugate is a view with a minus that its memory does not hold."""
    def view(*s):
        v = torch.complex(torch.ones(*s), torch.ones(*s)).conj().imag
        assert v.is_neg() and (v == -1).all()
        return v

    f, e = torch.ones, _experts()
    for call in (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), gate=view(3, 8)), lambda: ops.block_norm(f(3, 1), view(3, 1), f(1)),
                 lambda: ops.route(view(3, 1), 1), lambda: e(f(1, 8), torch.zeros(1, 1, dtype=torch.int32), view(1, 1))):
        with pytest.raises(ValueError, match="negated"):
            call()
    assert not no_device
    ops.block_norm(f(3, 8), f(3, 8), f(8), gate=view(3, 8).resolve_neg())


def test_optional_tensors_whose_memory_was_freed_are_refused(no_device, lib):  # noqa: F811
    """They have no address, which stands for an array that is not given: a bias or a gate would be left out without a word."""
    def freed(*s):
        t = torch.ones(*s)
        t.untyped_storage().resize_(0)
        return t

    f = torch.ones
    for call, name in ((lambda: ops.route(f(3, 8), 2, bias=freed(8)), "bias"), (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), gate=freed(3, 1)), "gate"),
                       (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), offset=freed(8)), "offset"),
                       (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), post_gain=freed(8)), "post_gain"),
                       (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), post_gain=f(8), post_offset=freed(8)), "post_offset")):
        with pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
            call()
    assert not no_device
    ops.block_norm(f(0, 8), f(0, 8), f(8), gate=f(0, 8))  # an empty one is a tensor


def test_optional_views_whose_memory_was_freed_are_refused(no_device, lib):  # noqa: F811
    """A view behind the storage's begin has an address without it."""
    def freed(n):
        t = torch.ones(2 * n)
        v = t[n:]
        t.untyped_storage().resize_(0)
        return v

    f = torch.ones
    for call, name in ((lambda: ops.route(f(3, 8), 2, bias=freed(8)), "bias"), (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), offset=freed(8)), "offset"),
                       (lambda: ops.block_norm(f(3, 8), f(3, 8), f(8), gate=freed(8)), "gate")):
        with pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
            call()
    assert not no_device
