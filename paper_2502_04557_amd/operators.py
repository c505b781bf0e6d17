"""The operators of include/sprinter.h on torch tensors: routing to experts, the experts' products, the norms around a block; a cache in pages,
the attention of drafted trees over it, and the adjustments of logits.

Argument marshalling only; every call runs the library's HIP kernels on the device and the current stream of its tensors, allocates its
outputs (and workspace) through torch and waits for nothing.  Options are plain numbers, no tensors.  What the library refuses raises
SprinterError, what is no tensor of the right type, shape or device, or no such number, ValueError.  There are no gradients: a tensor that
asks for one, or that carries a tangent of forward mode, is refused.
"""
from __future__ import annotations
import ctypes as C
from functools import lru_cache
from numbers import Integral, Real
import struct
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


def _memory(name, t):
    """The address of `t`, whose storage may have been freed, or a part of it (no address would stand for no tensor)."""
    at = t.data_ptr()
    if t.numel() > 0:
        last = t.storage_offset() + sum((n - 1) * d for n, d in zip(t.shape, t.stride()))
        if at == 0 or (last + 1) * t.element_size() > t.untyped_storage().nbytes():
            raise ValueError(f"{name}: a tensor without memory")
    return at


def _ptr(name, t):
    """The address of an optional tensor; freed storage is looked for here at a tenth of what _memory costs."""
    if t is None:
        return None
    at = t.data_ptr()
    return at if at and t.untyped_storage().nbytes() else _memory(name, t)


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
    _call("sprinter_route", dev, cfg[1], logits.data_ptr(), logits.stride(0), _ptr("bias", bias), T, ids.data_ptr(), weights.data_ptr())
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
    gate_at, gate_row, gate_col = None, 0, 0
    if gate is not None:
        _tensor("gate", gate, dev, torch.float32)
        gate_at = _ptr("gate", gate)
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
    _call("sprinter_block_norm", dev, cfg[1], h.data_ptr(), h.stride(0), y.data_ptr(), y.stride(0), _ptr("post_gain", post_gain), _ptr("post_offset", post_offset),
          gate_at, gate_row, gate_col, gain.data_ptr(), _ptr("offset", offset), T, h_out.data_ptr(), h_out.stride(0), out.data_ptr(), out.stride(0))
    if given:
        _written(h_out)
    return h_out, out


# ------------------------------------------------------------------------------------ a round of drafted trees over a cache in pages
PAIRS = {"halves": 0, "neighbours": 1}
Tensor = torch.Tensor

# The structs of include/sprinter.h, packed in one go: arguments by the dozen cost ctypes 0.1 us each.
_APPEND = struct.Struct("4i 2P Pq 3P P Pq Pq Pq Pq 4i")
_ATTEND = struct.Struct("4i 2P Pq 2P P Pq Pq PQ 2if 0Q")
_KEEP = struct.Struct("3i 2P Pq 2P Pq P")
_LOGITS = struct.Struct("4i Pq Pq P Pq 2P 3P P P Pq Pq Pq P 4i")


class CacheCfgC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_layer", "n_page", "page_size", "n_kv_head", "d_head")]


_native = None


def _asks():
    """The extension that looks tensors over (csrc/tensors.cpp).  Raises if it is not built."""
    global _native
    if _native is None:
        try:
            from . import _tensors
        except ImportError as e:
            raise RuntimeError("paper_2502_04557_amd/_tensors.so not found: build it first (python -m paper_2502_04557_amd.build)") from e
        _native = _tensors
    return _native


def _no(*args):
    return None


def _looks():
    """Its (rows, vector, arrays); inside a level of forward mode, whose tangents it does not see, everything takes the checks in Python."""
    n = _native or _asks()
    return (n.rows, n.vector, n.arrays) if forward_ad._current_level < 0 else (_no, _no, _no)


# What those say None of: the checks in Python, which raise, or let the uncommon (an empty tensor, one that asks for gradients where they are off) pass.
def _matrix(name, t, device, dtype, rows, cols):
    _rows(name, t, device, dtype, None if rows < 0 else rows, None if cols < 0 else cols)
    for what, n in zip(("rows", "columns"), t.shape):
        _int32(f"{name}'s {what}", n)
    return (_memory(name, t), t.stride(0), *t.shape)


def _column(name, t, device, dtype, n):
    _whole(name, t, device, dtype, n)
    return _memory(name, t)


def _layer(v):
    return v if type(v) is int and 0 <= v < 65536 else _int32("layer", v)


def _words(rows, visible, device, n):
    """The address of `visible` and the words of its rows."""
    if visible is None:
        return 0, 0
    at, ld, _, words = rows(visible, device, torch.int64, n, -1) or (0, -1, 0, 0)
    if ld != words or words < 1:
        words = visible.shape[1] if isinstance(visible, Tensor) and visible.dim() == 2 else 0
        _whole("visible", visible, device, torch.int64, n, max(1, words))
        at = _memory("visible", visible)
    return at, words


class PagedCache:
    """A cache in pages on two tensors of the caller's: keys, values [n_layer, n_page, n_kv_head, page_size, d_head], bfloat16 or float32.

    Slot s of sequence b is place s % page_size of page table[b, s // page_size] (table int32 [n_seq, n], entries outside the cache: no page).  page_size is a
    power of two in [8, 1024], d_head 64 or 128.  The tensors are written in place; the object keeps no state beside them.  Rows that `attend` reads and writes are
    16-byte aligned.

    A batch of trees: sequence b has lens[b] committed slots and the rows first[b] .. first[b + 1] - 1 as its drafted nodes (lens int32 [n_seq], first int32
    [n_seq + 1]), node i in slot lens[b] + i.  visible int64 [T, words]: bit j % 64 of word j // 64 says whether a row sees node j of its sequence,
    itself among them; None: the nodes up to itself (a decode step, a window of drafted tokens, a piece of a prompt)."""

    def __init__(self, keys, values):
        dev = _device(keys, "keys")
        if keys.dtype not in DTYPES or keys.dim() != 5:
            raise ValueError("keys: bfloat16 or float32 [n_layer, n_page, n_kv_head, page_size, d_head] is needed")
        shape = tuple(keys.shape)
        for name, t in (("keys", keys), ("values", values)):
            _whole(name, t, dev, keys.dtype, *shape)
            _memory(name, t)
        self._keys, self._values, self.device, self.dtype = keys, values, dev, keys.dtype
        self.n_layer, self.n_page, self.n_kv_head, self.page_size, self.d_head = shape
        self._cfg = CacheCfgC(DTYPES[keys.dtype], *(_int32("keys' sizes", shape[i]) for i in (0, 1, 3, 2, 4)))
        self._ref = C.byref(self._cfg)
        self._shape, self._elements = shape, keys.numel()
        self._need = {}

    def _arrays(self):
        """The addresses of keys and values: theirs of this call, as their memory may have moved or gone."""
        for name, t in (("keys", self._keys), ("values", self._values)):
            _whole(name, t, self.device, self.dtype, *self._shape)
        return _memory("keys", self._keys), _memory("values", self._values)

    @property
    def keys(self):
        return self._keys

    @property
    def values(self):
        return self._values

    def append(self, layer, keys, values, table, seq, slot, *, q=None, pos=None, freq=None, pairs="halves", q_out=None):
        """Writes the rows keys, values [T, n_kv_head * d_head] to slot[t] of sequence seq[t] (both int32 [T]); -> q turned, or None (sprinter_cache_append).

        With freq (float64 [n / 2]) the first n columns of each head of the keys and of q [T, n_head * d_head] are turned by the angles pos[t] * freq (pos int32
        [T], by default the slot), in the pairs (i, i + n / 2) ("halves") or (2 i, 2 i + 1) ("neighbours").  Rows are bfloat16 or float32, all of one
        type; what is written has the cache's.  A token of no sequence (-1) is padding.  q_out: where the turned q goes (q itself turns it in place)."""
        dev, d, i32 = self.device, self.d_head, torch.int32
        rows, vector, arrays = _looks()
        cache_keys, cache_values = arrays(self._keys, self._values, dev, self.dtype, self._elements) or self._arrays()
        dtype = keys.dtype if isinstance(keys, Tensor) else None
        if dtype not in DTYPES:
            raise ValueError("keys: bfloat16 or float32 rows are needed")
        width = self.n_kv_head * d
        k, ld_k, T, _ = rows(keys, dev, dtype, -1, width) or _matrix("keys", keys, dev, dtype, -1, width)
        v, ld_v, _, _ = rows(values, dev, dtype, T, width) or _matrix("values", values, dev, dtype, T, width)
        tab, ld_tab, n_seq, n_table = rows(table, dev, i32, -1, -1) or _matrix("table", table, dev, i32, -1, -1)
        seq_at = vector(seq, dev, i32, T) or _column("seq", seq, dev, i32, T)
        slot_at = vector(slot, dev, i32, T) or _column("slot", slot, dev, i32, T)
        pos_at = 0 if pos is None else vector(pos, dev, i32, T) or _column("pos", pos, dev, i32, T)
        n = freq_at = 0
        if freq is not None:
            n = freq.shape[0] if isinstance(freq, Tensor) and freq.dim() == 1 else 0
            freq_at = vector(freq, dev, torch.float64, n) or _column("freq", freq, dev, torch.float64, n)
        if pairs not in PAIRS:
            raise ValueError(f"pairs is one of {tuple(PAIRS)}")
        H = q_at = ld_q = to = ld_to = 0
        given = q_out is not None
        if q is not None:
            q_at, ld_q, _, wide = rows(q, dev, dtype, T, -1) or _matrix("q", q, dev, dtype, T, -1)
            H = wide // d
            if H < 1 or wide != H * d:
                raise ValueError(f"q: {wide} columns are no heads of {d}")
            if not given:
                q_out = _native.empty(T, wide, self.dtype, dev)
            to, ld_to, _, _ = rows(q_out, dev, self.dtype, T, wide) or _matrix("q_out", q_out, dev, self.dtype, T, wide)
        elif given:
            raise ValueError("q_out: there is no q")
        _call("sprinter_cache_append", dev, self._ref, _APPEND.pack(
            _layer(layer), n_seq, n_table, T, cache_keys, cache_values, tab, ld_tab, seq_at, slot_at, pos_at, freq_at, k, ld_k, v, ld_v, q_at, ld_q,
            to, ld_to, H, 2 * n, PAIRS[pairs], DTYPES[dtype]))
        if given:
            _native.written(self._keys, self._values, q_out)
        else:
            _native.written(self._keys, self._values)
        return q_out

    def attend(self, layer, q, table, lens, first, *, visible=None, scale=None, out=None):
        """q [T, n_head * d_head] of the cache's type -> y [T, n_head * d_head]: each node attends to the committed slots and to the nodes that it
        sees (sprinter_cache_attend).  scale: of the scores, by default d_head ** -0.5.  A row that sees nothing gives zeros; rows of no
        sequence are not written."""
        dev, dtype, i32 = self.device, self.dtype, torch.int32
        rows, vector, arrays = _looks()
        keys, values = arrays(self._keys, self._values, dev, self.dtype, self._elements) or self._arrays()
        q_at, ld_q, T, width = rows(q, dev, dtype, -1, -1) or _matrix("q", q, dev, dtype, -1, -1)
        H = width // self.d_head
        if H < 1 or width != H * self.d_head:
            raise ValueError(f"q: {width} columns are no heads of {self.d_head}")
        tab, ld_tab, n_seq, n_table = rows(table, dev, i32, -1, -1) or _matrix("table", table, dev, i32, -1, -1)
        lens_at = vector(lens, dev, i32, n_seq) or _column("lens", lens, dev, i32, n_seq)
        first_at = vector(first, dev, i32, n_seq + 1) or _column("first", first, dev, i32, n_seq + 1)
        seen, words = _words(rows, visible, dev, T)
        given = out is not None
        if not given:
            out = _native.empty(T, width, dtype, dev)
        to, ld_to, _, _ = rows(out, dev, dtype, T, width) or _matrix("out", out, dev, dtype, T, width)
        scale = self.d_head ** -0.5 if scale is None else float(_number("scale", scale))
        if 3.4e38 < abs(scale) < float("inf"):
            raise ValueError(f"scale: {scale} is beyond float32")
        need = self._workspace(H, n_seq, n_table, T)
        work = _native.empty(1, need, torch.uint8, dev) if need else None
        _call("sprinter_cache_attend", dev, self._ref, _ATTEND.pack(
            _layer(layer), n_seq, n_table, T, keys, values, tab, ld_tab, lens_at, first_at, seen, q_at, ld_q, to, ld_to,
            0 if work is None else work.data_ptr(), need, words, H, scale))
        if given:
            _native.written(out)
        return out

    def _workspace(self, H, n_seq, n_table, T):
        n = self._need.get((H, n_seq, n_table, T))
        if n is None:
            v = C.c_size_t(0)
            rc = _entry("sprinter_cache_attend_bytes")(self._ref, _int32("heads", H), n_seq, _int32("table's columns", n_table), T, C.byref(v))
            if rc:
                raise SprinterError(rc, _lib.sprinter_last_error(None).decode())
            if len(self._need) >= 4096:
                self._need.clear()
            n = self._need[H, n_seq, n_table, T] = v.value
        return n

    def keep(self, table, lens, first, path, n_keep):
        """Slot lens[b] + path[b, j] -> slot lens[b] + j in every layer, j < n_keep[b] (path int32 [n_seq, n], nodes in ascending order; n_keep int32
        [n_seq]): the accepted nodes become the next committed slots (sprinter_cache_keep).  lens is the caller's to advance."""
        dev, i32 = self.device, torch.int32
        rows, vector, arrays = _looks()
        keys, values = arrays(self._keys, self._values, dev, self.dtype, self._elements) or self._arrays()
        tab, ld_tab, n_seq, n_table = rows(table, dev, i32, -1, -1) or _matrix("table", table, dev, i32, -1, -1)
        lens_at = vector(lens, dev, i32, n_seq) or _column("lens", lens, dev, i32, n_seq)
        first_at = vector(first, dev, i32, n_seq + 1) or _column("first", first, dev, i32, n_seq + 1)
        path_at, ld_path, _, n_path = rows(path, dev, i32, n_seq, -1) or _matrix("path", path, dev, i32, n_seq, -1)
        keep_at = vector(n_keep, dev, i32, n_seq) or _column("n_keep", n_keep, dev, i32, n_seq)
        _call("sprinter_cache_keep", dev, self._ref, _KEEP.pack(n_seq, n_table, n_path, keys, values, tab, ld_tab, lens_at, first_at,
                                                                path_at, ld_path, keep_at))
        _native.written(self._keys, self._values)


def adjust_logits(logits, first=None, *, tokens=None, n_token=None, n_prompt=None, repetition=None, presence=None, frequency=None, draft=None,
                  visible=None, bias_ids=None, bias=None, mask=None, mask_row=None, out=None):
    """logits [T, V] float32 or bfloat16 -> penalties for the tokens of each row, biases and a mask applied (sprinter_adjust_logits).

    Rows first[b] .. first[b + 1] - 1 are the nodes of sequence b (None: row t is sequence t).  tokens int32 [n_seq, n] with n_token, n_prompt int32 [n_seq]: a
    sequence's tokens, how many there are (None: n), and how many of them are its prompt (None: none); draft int32 [T] with visible, as for
    PagedCache: the drafted tokens, of which a row's own are those that it sees.  repetition divides positive logits of a row's tokens and multiplies others;
    frequency times how often a token was generated, and presence if it was, are subtracted (float32 [n_seq]).  bias_ids int32, bias float32
    [n_seq, n]: biases of tokens (an id outside the vocabulary is padding, the last of equal ids counts).  mask int32 [n, ceil(V / 32)], mask_row
    int32 [T]: row t may take the tokens whose bits mask[mask_row[t]] has, the others become -inf (-1: all allowed; None: mask t).  out: logits itself changes them in
    place."""
    dev = _device(logits, "logits")
    if logits.dtype not in DTYPES:
        raise ValueError("logits: bfloat16 or float32 is needed")
    dtype, f32, i32 = logits.dtype, torch.float32, torch.int32
    rows, vector, _ = _looks()
    at, ld, T, V = rows(logits, dev, dtype, -1, -1) or _matrix("logits", logits, dev, dtype, -1, -1)
    n_seq, first_at = T, 0
    if first is not None:
        n_seq = first.shape[0] - 1 if isinstance(first, Tensor) and first.dim() == 1 else -1
        if n_seq < 0:
            raise ValueError("first: an int32 vector [n_seq + 1] is needed")
        first_at = vector(first, dev, i32, n_seq + 1) or _column("first", first, dev, i32, n_seq + 1)
    seen, words = _words(rows, visible, dev, T)
    many = 0 if n_token is None else vector(n_token, dev, i32, n_seq) or _column("n_token", n_token, dev, i32, n_seq)
    asked = 0 if n_prompt is None else vector(n_prompt, dev, i32, n_seq) or _column("n_prompt", n_prompt, dev, i32, n_seq)
    rep = 0 if repetition is None else vector(repetition, dev, f32, n_seq) or _column("repetition", repetition, dev, f32, n_seq)
    pre = 0 if presence is None else vector(presence, dev, f32, n_seq) or _column("presence", presence, dev, f32, n_seq)
    frq = 0 if frequency is None else vector(frequency, dev, f32, n_seq) or _column("frequency", frequency, dev, f32, n_seq)
    drafted = 0 if draft is None else vector(draft, dev, i32, T) or _column("draft", draft, dev, i32, T)
    row = 0 if mask_row is None else vector(mask_row, dev, i32, T) or _column("mask_row", mask_row, dev, i32, T)
    tok = ld_tok = n_tokens = ids = ld_ids = add = ld_add = n_bias = bits = ld_bits = n_mask = 0
    if tokens is not None:
        tok, ld_tok, _, n_tokens = rows(tokens, dev, i32, n_seq, -1) or _matrix("tokens", tokens, dev, i32, n_seq, -1)
        if n_tokens == 0:                                # (no history: an empty tensor has no address)
            tok = many = asked = 0
    if bias is not None or bias_ids is not None:
        ids, ld_ids, _, n_bias = rows(bias_ids, dev, i32, n_seq, -1) or _matrix("bias_ids", bias_ids, dev, i32, n_seq, -1)
        add, ld_add, _, _ = rows(bias, dev, f32, n_seq, n_bias) or _matrix("bias", bias, dev, f32, n_seq, n_bias)
    if mask is not None:
        bits, ld_bits, n_mask, _ = rows(mask, dev, i32, -1, (V + 31) // 32) or _matrix("mask", mask, dev, i32, -1, (V + 31) // 32)
        if n_mask == 0:
            if mask_row is None and T > 0:
                raise ValueError(f"mask: {T} rows without mask_row, and no masks")
            bits = row = 0
    given = out is not None
    if not given:
        out = _native.empty(T, V, dtype, dev)
    to, ld_to, _, _ = rows(out, dev, dtype, T, V) or _matrix("out", out, dev, dtype, T, V)
    _call("sprinter_adjust_logits", dev, _LOGITS.pack(
        DTYPES[dtype], T, V, n_seq, at, ld, to, ld_to, first_at, tok, ld_tok, many, asked, rep, pre, frq, drafted, seen, ids, ld_ids, add, ld_add, bits, ld_bits, row,
        n_tokens, words, n_bias, n_mask))
    if given:
        _native.written(out)
    return out
