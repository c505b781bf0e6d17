"""The operators of include/sprinter.h on torch tensors: routing to experts, the experts' products, the norms around a block.

Argument marshalling only; every call runs the library's HIP kernels on the device and the current stream of its tensors, allocates its
outputs (and workspace) through torch and waits for nothing.  Options are plain numbers, no tensors.  What the library refuses raises
SprinterError, what is no tensor of the right type, shape or device, or no such number, ValueError.  There are no gradients: a tensor that
asks for one, or that carries a tangent of forward mode, is refused.
"""
from __future__ import annotations
import ctypes as C
from functools import lru_cache
from numbers import Integral, Real
import torch
import torch.autograd.forward_ad as forward_ad

from .binding import F32, BF16, GROUP_SCORES, SCORES, RouteCfgC, SprinterError, load_library

NORMS = {"layer": 0, "rms": 1}
DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


class ExpertsCfgC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_expert", "d_model", "d_ff")]


class BlockNormCfgC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "kind", "d")] + [("eps", C.c_float), ("scale", C.c_float)]


# The smallest kernels run for 2 - 4 us, so the host's side counts: raw handles instead of torch.cuda.Stream objects, no generators.
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_lib = None


def _entry(name):
    global _lib
    if _lib is None:
        _lib = load_library()
    return getattr(_lib, name)


def _call(name, device, *args):
    """One entry point on `device` and its current stream (the last argument of them all)."""
    index = device.index
    if _current_device() == index:
        rc = _entry(name)(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            rc = _entry(name)(*args, _raw_stream(index))
    if rc != 0:
        raise SprinterError(rc, _lib.sprinter_last_error(None).decode())


def _tensor(name, t, device, dtype):
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name}: a {dtype} tensor on {device} is needed")
    if t.is_neg():                                       # (its memory holds the values before the minus)
        raise ValueError(f"{name}: a negated view; resolve_neg it")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: gradients are not computed here; detach it")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name}: tangents are not computed here; unpack it")


def _rows(name, t, device, dtype, rows, cols):
    """A matrix whose rows may lie apart; rows, cols: None for any."""
    _tensor(name, t, device, dtype)
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name}: shape {tuple(shape)}, expected [{rows or 'any'}, {cols or 'any'}]")
    if shape[0] >= 2 ** 31:
        raise ValueError(f"{name}: {shape[0]} rows are more than 32 bits hold")
    if not t.is_contiguous() and shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row are not adjacent")


def _whole(name, t, device, dtype, *shape):
    """A contiguous array of this shape."""
    _tensor(name, t, device, dtype)
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {list(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")


def _device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a tensor on a GPU is needed")
    return t.device


def _int32(name, v):
    """A whole number that the library's 32 bits hold (ctypes would cut others off and pass what is left)."""
    if not isinstance(v, Integral) or not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name}: {v!r} is no whole number of 32 bits")
    return v


def _number(name, v):
    """A plain number: the configurations are kept by their values, and a tensor's can change while it stays the same key."""
    if not isinstance(v, Real):
        raise ValueError(f"{name}: {type(v).__name__} is no plain number")
    return v


_written = torch.autograd.graph.increment_version          # what autograd has kept of a tensor that is written in place is out of date


def _ptr(t):
    return None if t is None else t.data_ptr()


@lru_cache(maxsize=256)
def _route_cfg(n_expert, top_k, score, n_group, top_group, group_score, renormalize, n_shared, scale):
    if score not in SCORES or group_score not in GROUP_SCORES:
        raise ValueError(f"score is one of {tuple(SCORES)}, group_score one of {tuple(GROUP_SCORES)}")
    for name, v in (("logits' columns", n_expert), ("top_k", top_k), ("n_group", n_group), ("top_group", top_group), ("n_shared", n_shared),
                    ("renormalize", renormalize)):
        _int32(name, v)
    c = RouteCfgC(n_expert, top_k, SCORES[score], n_group, top_group, GROUP_SCORES[group_score], bool(renormalize), n_shared, _number("scale", scale))
    return c, C.byref(c)


def route(logits, top_k, *, score="softmax", bias=None, n_group=1, top_group=1, group_score="max", renormalize=True, scale=1.0,
          n_shared=0):
    """logits [T, E] float32 -> (ids int32, weights float32), both [T, top_k + n_shared] (sprinter_route)."""
    dev = _device(logits, "logits")
    _rows("logits", logits, dev, torch.float32, None, None)
    T, E = logits.shape
    if bias is not None:
        _whole("bias", bias, dev, torch.float32, E)
    if type(renormalize) is not bool and not isinstance(renormalize, torch.Tensor):
        renormalize = bool(renormalize)                  # (numpy's, which is no Integral)
    cfg = _route_cfg(E, top_k, score, n_group, top_group, group_score, renormalize, n_shared, scale)
    n = max(0, top_k + n_shared)
    ids = torch.empty(T, n, dtype=torch.int32, device=dev)
    weights = torch.empty(T, n, dtype=torch.float32, device=dev)
    _call("sprinter_route", dev, cfg[1], logits.data_ptr(), logits.stride(0), _ptr(bias), T, ids.data_ptr(), weights.data_ptr())
    return ids, weights


class Experts:
    """A set of experts on one device: gate, up [E, d_ff, d_model], down [E, d_model, d_ff], bfloat16 or float32.

    bfloat16 weights are laid out once here (on the current stream) and may go afterwards; float32 ones are kept and read as they are.

    Arithmetic of bfloat16: the framework's for its bfloat16 models, matrix products of float16 operands with float32 sums.  Weights below 2^-14 lose
    bits (below 2^-25: all), rows and hidden values silu(Wg x) * (Wu x) above 65504 become infinite, and hidden values are rounded to
    2^-11, which adds less than 1 % to the mean distance of the result, a bfloat16, from 64 bits.  float32: float32 throughout."""

    def __init__(self, gate, up, down):
        dev = _device(gate, "gate")
        if gate.dtype not in DTYPES or gate.dim() != 3:
            raise ValueError("gate: bfloat16 or float32 [n_expert, d_ff, d_model] is needed")
        E, ff, d = gate.shape
        for name, t, shape in (("gate", gate, (E, ff, d)), ("up", up, (E, ff, d)), ("down", down, (E, d, ff))):
            _whole(name, t, dev, gate.dtype, *shape)
        self.device, self.dtype = dev, gate.dtype
        self.n_expert, self.d_ff, self.d_model = E, ff, d
        self._cfg = ExpertsCfgC(DTYPES[gate.dtype], _int32("n_expert", E), _int32("d_model", d), _int32("d_ff", ff))
        self._ref = C.byref(self._cfg)
        self._need = {}
        n_up, n_down, _ = self._bytes(0, 1)
        if gate.dtype == torch.float32:
            self._weights = (gate, up, down)
        else:
            self._weights = tuple(torch.empty(n, dtype=torch.uint8, device=dev) for n in (n_up, n_up, n_down))
            for i, t in enumerate((gate, up, down)):
                _call("sprinter_experts_pack", dev, self._ref, int(i == 2), t.data_ptr(), self._weights[i].data_ptr())
        self._ptrs = tuple(t.data_ptr() for t in self._weights)

    def _bytes(self, rows, top_k):
        n = self._need.get((rows, top_k))
        if n is None:
            _int32("rows", rows)
            _int32("ids' columns", top_k)
            v = [C.c_size_t(0) for _ in range(3)]
            rc = _entry("sprinter_experts_bytes")(self._ref, rows, top_k, *(C.byref(x) for x in v))
            if rc:
                raise SprinterError(rc, _lib.sprinter_last_error(None).decode())
            if len(self._need) >= 4096:
                self._need.clear()
            n = self._need[rows, top_k] = tuple(x.value for x in v)
        return n

    def __call__(self, x, ids, weights, out=None):
        """x [T, d_model] -> y [T, d_model] of its type; ids int32, weights float32 [T, top_k] as `route` gives them (sprinter_experts)."""
        dev = self.device
        _rows("x", x, dev, self.dtype, None, self.d_model)
        T = x.shape[0]
        k = ids.shape[1] if isinstance(ids, torch.Tensor) and ids.dim() == 2 else 0
        _whole("ids", ids, dev, torch.int32, T, k)
        _whole("weights", weights, dev, torch.float32, T, k)
        given = out is not None
        if given:
            _rows("out", out, dev, self.dtype, T, self.d_model)
        else:
            out = torch.empty(T, self.d_model, dtype=self.dtype, device=dev)
        need = self._bytes(T, k)[2]
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        _call("sprinter_experts", dev, self._ref, *self._ptrs, x.data_ptr(), x.stride(0), ids.data_ptr(), weights.data_ptr(), T, k,
              out.data_ptr(), out.stride(0), work.data_ptr(), need)
        if given:
            _written(out)
        return out


@lru_cache(maxsize=256)
def _norm_cfg(dtype, kind, d, eps, scale):
    if dtype not in DTYPES or kind not in NORMS:
        raise ValueError(f"y is bfloat16 or float32, kind one of {tuple(NORMS)}")
    c = BlockNormCfgC(DTYPES[dtype], NORMS[kind], _int32("d", d), _number("eps", eps), _number("scale", scale))
    return c, C.byref(c)


def block_norm(h, y, gain, *, offset=None, post_gain=None, post_offset=None, gate=None, scale=1.0, eps=1e-5, kind="rms", h_out=None):
    """u = norm(y) (or y without post_gain), h' = h + scale * gate * u, out = norm(h') -> (h', out) (sprinter_block_norm).

    h [T, d] float32, y [T, d] bfloat16 or float32; gate float32 of any shape that broadcasts to [T, d].  h_out: where h' goes (h itself
    updates it in place); by default a new tensor."""
    dev = _device(h, "h")
    _rows("h", h, dev, torch.float32, None, None)
    T, d = h.shape
    if not isinstance(y, torch.Tensor):
        raise ValueError("y: a tensor is needed")
    cfg = _norm_cfg(y.dtype, kind, d, eps, scale)
    _rows("y", y, dev, y.dtype, T, d)
    _whole("gain", gain, dev, torch.float32, d)
    if offset is not None:
        _whole("offset", offset, dev, torch.float32, d)
    if post_gain is not None:
        _whole("post_gain", post_gain, dev, torch.float32, d)
    if post_offset is not None:
        _whole("post_offset", post_offset, dev, torch.float32, d)
    gate_row = gate_col = 0
    if gate is not None:
        _tensor("gate", gate, dev, torch.float32)
        try:
            gate = gate.expand(T, d)
        except RuntimeError as e:
            raise ValueError(f"gate: shape {tuple(gate.shape)} does not broadcast to {(T, d)}") from e
        gate_row, gate_col = gate.stride()
    given = h_out is not None
    if given:
        _rows("h_out", h_out, dev, torch.float32, T, d)
    else:
        h_out = torch.empty(T, d, dtype=torch.float32, device=dev)
    out = torch.empty(T, d, dtype=y.dtype, device=dev)
    _call("sprinter_block_norm", dev, cfg[1], h.data_ptr(), h.stride(0), y.data_ptr(), y.stride(0), _ptr(post_gain), _ptr(post_offset),
          _ptr(gate), gate_row, gate_col, gain.data_ptr(), _ptr(offset), T, h_out.data_ptr(), h_out.stride(0), out.data_ptr(), out.stride(0))
    if given:
        _written(h_out)
    return h_out, out
