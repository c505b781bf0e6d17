"""What the operators' entry points refuse, on the CPU: arguments are checked before any device work, so addresses that nobody may
read stand in for device arrays."""
import ctypes as C
import numpy as np
import pytest
import torch
from test_abi_cpu import lib  # noqa: F401
from paper_2502_04557_amd import operators as ops

A = 0x10000          # an aligned address
NULL, CONFIG, WORKSPACE, RANGE = -1, -2, -3, -5


def _refused(lib, rc, code, word):  # noqa: F811
    assert rc == code and word in lib.sprinter_last_error(None).decode(), (rc, lib.sprinter_last_error(None))


def test_layouts():
    assert C.sizeof(ops.RouteCfgC) == 36 and C.sizeof(ops.ExpertsCfgC) == 16 and C.sizeof(ops.BlockNormCfgC) == 20


@pytest.mark.parametrize("change, word", [
    (dict(n_expert=0), "n_expert"), (dict(n_expert=1025), "n_expert"), (dict(top_k=0), "top_k"), (dict(top_k=9), "top_k"),
    (dict(n_expert=64, top_k=49), "top_k"), (dict(score=2), "score"), (dict(n_group=0), "n_group"), (dict(n_group=3), "n_group"),
    (dict(n_expert=128, n_group=128), "n_group"), (dict(top_group=2), "top_group"), (dict(n_group=4, top_group=1, top_k=3), "top_group"),
    (dict(n_group=4, top_group=0), "top_group"), (dict(group_score=2), "group_score"), (dict(n_shared=-1), "n_shared"),
    (dict(n_shared=17), "n_shared"), (dict(scale=0.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale")])
def test_route_configuration(lib, change, word):  # noqa: F811
    v = dict(n_expert=8, top_k=2, score=0, n_group=1, top_group=1, group_score=0, renormalize=1, n_shared=0, scale=1.0)
    v.update(change)
    _refused(lib, lib.sprinter_route(C.byref(ops.RouteCfgC(**v)), A, 1024, None, 4, A, A, None), CONFIG, word)


def test_route_arguments(lib):  # noqa: F811
    c = C.byref(ops.RouteCfgC(8, 2, 0, 1, 1, 0, 1, 0, 1.0))
    _refused(lib, lib.sprinter_route(None, A, 8, None, 1, A, A, None), NULL, "configuration")
    for args in ((None, 8, None, 1, A, A), (A, 8, None, 1, None, A), (A, 8, None, 1, A, None)):
        _refused(lib, lib.sprinter_route(c, *args, None), NULL, "NULL array")
    _refused(lib, lib.sprinter_route(c, A, 8, None, -1, A, A, None), RANGE, "-1 rows")
    _refused(lib, lib.sprinter_route(c, A, 8, None, (1 << 23) + 1, A, A, None), RANGE, "rows")
    _refused(lib, lib.sprinter_route(c, A, 7, None, 2, A, A, None), RANGE, "8 logits")
    _refused(lib, lib.sprinter_route(c, A + 2, 8, None, 2, A, A, None), RANGE, "aligned")
    assert lib.sprinter_route(c, None, 0, None, 0, None, None, None) == 0


@pytest.mark.parametrize("v, word", [((2, 8, 64, 64), "dtype"), ((1, 0, 64, 64), "n_expert"), ((1, 1025, 64, 64), "n_expert"),
                                     ((1, 8, 60, 64), "d_model"), ((1, 8, 0, 64), "d_model"), ((1, 8, 8200, 64), "d_model"),
                                     ((0, 8, 64, 12), "d_ff"), ((0, 8, 64, 65544), "d_ff")])
def test_experts_configuration(lib, v, word):  # noqa: F811
    c = C.byref(ops.ExpertsCfgC(*v))
    _refused(lib, lib.sprinter_experts_bytes(c, 1, 1, None, None, None), CONFIG, word)
    _refused(lib, lib.sprinter_experts_pack(c, 0, A, A, None), CONFIG, word)
    _refused(lib, lib.sprinter_experts(c, A, A, A, A, 64, A, A, 1, 1, A, 64, A, 1 << 40, None), CONFIG, word)


def test_experts_arguments(lib):  # noqa: F811
    cfg = ops.ExpertsCfgC(1, 8, 64, 128)
    c = C.byref(cfg)
    need = C.c_size_t(0)
    up, down = C.c_size_t(0), C.c_size_t(0)
    assert lib.sprinter_experts_bytes(c, 4, 2, C.byref(up), C.byref(down), C.byref(need)) == 0
    assert up.value == down.value == 8 * 64 * 128 * 2 and need.value > 8 * 128 * 2
    good = dict(gate=A, up=A, down=A, x=A, ldx=64, ids=A, w=A, rows=4, k=2, y=A, ldy=64, ws=A, n=need.value)

    def call(**kw):
        return lib.sprinter_experts(c, *{**good, **kw}.values(), None)

    for name in ("gate", "up", "down", "x", "ids", "w", "y", "ws"):
        _refused(lib, call(**{name: None}), NULL, "NULL array")
    for name in ("gate", "up", "down", "x", "y"):
        _refused(lib, call(**{name: A + 8}), RANGE, "16-byte")
    _refused(lib, call(ids=A + 2), RANGE, "aligned")
    _refused(lib, call(ldx=56), RANGE, "columns")
    _refused(lib, call(ldy=63), RANGE, "columns")
    _refused(lib, call(ldx=68), RANGE, "16-byte")
    _refused(lib, call(rows=-1), RANGE, "rows")
    _refused(lib, call(k=0), RANGE, "top_k")
    _refused(lib, call(k=65), RANGE, "top_k")
    _refused(lib, call(rows=1 << 20), RANGE, "more than")
    _refused(lib, call(n=need.value - 1), WORKSPACE, "needed")
    _refused(lib, call(ws=A + 128), WORKSPACE, "256-byte")
    assert call(rows=0, x=None) == 0
    _refused(lib, lib.sprinter_experts(None, *good.values(), None), NULL, "configuration")
    _refused(lib, lib.sprinter_experts_pack(c, 0, None, A, None), NULL, "NULL array")
    _refused(lib, lib.sprinter_experts_pack(c, 1, A, A + 4, None), RANGE, "16-byte")
    _refused(lib, lib.sprinter_experts_pack(C.byref(ops.ExpertsCfgC(0, 8, 64, 128)), 0, A, A, None), CONFIG, "bf16")


def test_workspace_holds_every_row_of_the_largest_call(lib):  # noqa: F811
    """One slot per pair at least, sizes beyond 32 bits among them."""
    n = C.c_size_t(0)
    for dtype, es in ((0, 4), (1, 2)):
        c = C.byref(ops.ExpertsCfgC(dtype, 1024, 8192, 65536))
        assert lib.sprinter_experts_bytes(c, 1 << 14, 64, None, None, C.byref(n)) == 0
        assert n.value > (1 << 20) * (65536 * es + 8192 * 4)


@pytest.mark.parametrize("v, word", [((3, 1, 64, 1e-5, 1.0), "dtype"), ((1, 2, 64, 1e-5, 1.0), "kind"), ((1, 1, 0, 1e-5, 1.0), "d 0"),
                                     ((1, 1, 16385, 1e-5, 1.0), "16384"), ((1, 1, 64, -1.0, 1.0), "eps"), ((1, 1, 64, 1e-5, float("nan")), "scale")])
def test_block_norm_configuration(lib, v, word):  # noqa: F811
    c = C.byref(ops.BlockNormCfgC(*v))
    _refused(lib, lib.sprinter_block_norm(c, A, 64, A, 64, None, None, None, 0, 0, A, None, 1, A, 64, A, 64, None), CONFIG, word)


def test_block_norm_arguments(lib):  # noqa: F811
    c = C.byref(ops.BlockNormCfgC(1, 1, 64, 1e-5, 1.0))
    good = dict(h=A, ldh=64, y=A, ldy=64, pg=None, pb=None, gate=None, gr=0, gc=0, g=A, b=None, rows=2, ho=A, ldho=64, out=A, ldo=64)

    def call(**kw):
        return lib.sprinter_block_norm(c, *{**good, **kw}.values(), None)

    for name in ("h", "y", "g", "ho", "out"):
        _refused(lib, call(**{name: None}), NULL, "NULL array")
    _refused(lib, call(pb=A), NULL, "post_offset")
    for name in ("ldh", "ldy", "ldho", "ldo"):
        _refused(lib, call(**{name: 63}), RANGE, "closer")
    _refused(lib, call(gate=A, gr=-1), RANGE, "stride")
    _refused(lib, call(h=A + 2), RANGE, "aligned")
    _refused(lib, call(y=A + 1), RANGE, "aligned")
    _refused(lib, call(rows=-3), RANGE, "rows")
    _refused(lib, call(rows=(1 << 23) + 1), RANGE, "rows")
    assert call(rows=0, h=None) == 0


def test_tensors_that_are_none_of_a_gpu():
    with pytest.raises(ValueError, match="GPU"):
        ops.route(torch.zeros(2, 8), 2)
    with pytest.raises(ValueError, match="GPU"):
        ops.Experts(torch.zeros(2, 8, 8), torch.zeros(2, 8, 8), torch.zeros(2, 8, 8))
    with pytest.raises(ValueError, match="GPU"):
        ops.block_norm(torch.zeros(2, 8), torch.zeros(2, 8), torch.zeros(8))
    with pytest.raises(ValueError):
        ops.route(np.zeros((2, 8)), 2)


# ------------------------------------------------------------------------------------------ contexts with described blocks
@pytest.mark.parametrize("which", ["draft", "target"])
@pytest.mark.parametrize("change, word", [
    (dict(post_norm=2), "post_norm"), (dict(gate=-1), "gate"), (dict(route_bias=2), "route_bias"), (dict(residual_scale=float("nan")), "residual_scale"),
    (dict(d_expert=0), "d_expert"), (dict(d_expert=12), "d_expert"), (dict(d_expert=65544), "d_expert"), (dict(top_k=0), "top_k"),
    (dict(n_expert=1024, n_shared=1), "experts"), (dict(n_expert=-1), "n_expert"), (dict(scale=-1.0), "scale")])
def test_block_configuration(lib, which, change, word):  # noqa: F811
    import workloads as W
    from paper_2502_04557_amd import binding
    cfg = W.mini_config("llama")
    b = binding.blocks_to_c(W.mini_config("experts").target)
    for k, v in change.items():
        setattr(b.route if hasattr(b.route, k) else b, k, v)
    c = binding.cfg_to_c(cfg)
    n, ctx = C.c_size_t(0), C.c_void_p(None)
    pair = [C.byref(b), None] if which == "draft" else [None, C.byref(b)]
    for rc in (lib.sprinter_blocks_workspace_bytes(C.byref(c), *pair, C.byref(n)),
               lib.sprinter_create_blocks(C.byref(c), *pair, A, 1 << 40, None, C.byref(ctx))):
        _refused(lib, rc, CONFIG, word)
        assert which in lib.sprinter_last_error(None).decode()


def test_blocks_need_a_llama_model_and_their_workspace(lib):  # noqa: F811
    import workloads as W
    from paper_2502_04557_amd import binding
    b = binding.blocks_to_c(W.mini_config("experts").target)
    n, plain, ctx = C.c_size_t(0), C.c_size_t(0), C.c_void_p(None)
    c = binding.cfg_to_c(W.mini_config("gpt"))
    _refused(lib, lib.sprinter_blocks_workspace_bytes(C.byref(c), C.byref(b), None, C.byref(n)), CONFIG, "LLaMA")
    c = binding.cfg_to_c(W.mini_config("llama"))
    assert lib.sprinter_workspace_bytes(C.byref(c), C.byref(plain)) == 0
    assert lib.sprinter_blocks_workspace_bytes(C.byref(c), None, None, C.byref(n)) == 0 and n.value == plain.value
    assert lib.sprinter_blocks_workspace_bytes(C.byref(c), None, C.byref(b), C.byref(n)) == 0 and n.value > plain.value
    _refused(lib, lib.sprinter_create_blocks(C.byref(c), None, C.byref(b), A, n.value - 1, None, C.byref(ctx)), WORKSPACE, "needed")
    assert lib.sprinter_blocks_workspace_bytes(C.byref(c), None, None, None) == NULL
    with pytest.raises(ValueError, match="workspace of their own"):
        binding.Sprinter(W.mini_config("experts"), static_workspace=True)
