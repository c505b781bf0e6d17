"""What the entry points of the cache in pages and of the adjustments of logits refuse, on the CPU: arguments are checked before any device
work, so addresses that nobody may read stand in for device arrays."""
import ctypes as C
import pytest
import torch
from test_abi_cpu import lib  # noqa: F401
from test_operators_arguments import no_device  # noqa: F401
from paper_2502_04557_amd import operators as ops

A = 0x10000          # an aligned address
NULL, CONFIG, WORKSPACE, RANGE = -1, -2, -3, -5
CFG = dict(dtype=1, n_layer=2, n_page=10, page_size=16, n_kv_head=2, d_head=64)


def _refused(lib, rc, code, word):  # noqa: F811
    assert rc == code and word in lib.sprinter_last_error(None).decode(), (rc, lib.sprinter_last_error(None))


def _cfg(**kw):
    return C.byref(ops.CacheCfgC(*{**CFG, **kw}.values()))


APPEND = dict(layer=0, n_seq=3, n_table=4, T=5, keys=A, values=A, table=A, ldt=4, seq=A, slot=A, pos=None, freq=A, k=A, ldk=128, v=A, ldv=128, q=A, ldq=256, qo=A,
              ldqo=256, H=4, n=64, pairs=0, type=1)
ATTEND = dict(layer=0, n_seq=3, n_table=4, T=5, keys=A, values=A, table=A, ldt=4, lens=A, first=A, vis=A, q=A, ldq=256, y=A, ldy=256, work=A, bytes=1 << 40, words=1, H=4,
              scale=0.125)
KEEP = dict(n_seq=3, n_table=4, n_path=4, keys=A, values=A, table=A, ldt=4, lens=A, first=A, path=A, ldp=4, n_keep=A)
LOGITS = dict(dtype=0, n_rows=3, vocab=100, n_seq=3, logits=A, ld_logits=100, out=A, ld_out=100, first=A, tokens=A, ld_tokens=50, n_token=A, n_prompt=A,
              repetition=A, presence=A, frequency=A, draft=A, visible=A, bias_ids=A, ld_bias_ids=8, bias=A, ld_bias=8, mask=A, ld_mask=4, mask_row=A,
              n_tokens=50, n_words=1, n_bias=8, n_mask=2)


def _packed(layout, good, kw):
    assert not set(kw) - set(good)
    return layout.pack(*(0 if v is None else v for v in {**good, **kw}.values()))


def _append(lib, cfg=None, **kw):  # noqa: F811
    return lib.sprinter_cache_append(cfg or _cfg(), _packed(ops._APPEND, APPEND, kw), None)


def _attend(lib, cfg=None, **kw):  # noqa: F811
    return lib.sprinter_cache_attend(cfg or _cfg(), _packed(ops._ATTEND, ATTEND, kw), None)


def _keep(lib, cfg=None, **kw):  # noqa: F811
    return lib.sprinter_cache_keep(cfg or _cfg(), _packed(ops._KEEP, KEEP, kw), None)


def _logits(lib, **kw):  # noqa: F811
    return lib.sprinter_adjust_logits(_packed(ops._LOGITS, LOGITS, kw), None)


def test_layouts():
    """The structs as sprinter.h has them (their sizes are asserted where the library is compiled), field by field."""
    import os
    import re
    assert C.sizeof(ops.CacheCfgC) == 24
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sprinter.h")).read()
    for name, layout, size in (("append", ops._APPEND, 160), ("attend", ops._ATTEND, 136), ("keep", ops._KEEP, 88), ("logits", ops._LOGITS, 200)):
        body = re.search(r"typedef struct \{([^}]*)\} sprinter_%s;" % name, hdr).group(1)
        codes = ""
        for line in body.split(";"):
            words = line.replace("const ", "").split()
            if not words:
                continue
            kind, names = words[0], " ".join(words[1:]).split(",")
            codes += "".join("P" if "*" in n or kind.endswith("*") else {"int32_t": "i", "int64_t": "q", "uint64_t": "Q", "float": "f"}[kind] for n in names)
        given = re.sub(r"(\d+)(\w)", lambda m: m.group(2) * int(m.group(1)), layout.format.replace(" ", ""))
        assert given == codes and layout.size == size, (name, given, codes, layout.size)


@pytest.mark.parametrize("change, word", [(dict(dtype=2), "dtype"), (dict(n_layer=0), "n_layer"), (dict(n_page=0), "n_page"), (dict(page_size=4), "page_size"),
                                          (dict(page_size=24), "page_size"), (dict(page_size=2048), "page_size"), (dict(page_size=-16), "page_size"),
                                          (dict(n_kv_head=0), "n_kv_head"), (dict(n_kv_head=1025), "n_kv_head"), (dict(d_head=96), "d_head"), (dict(d_head=256), "d_head"),
                                          (dict(n_layer=65536), "n_layer")])
def test_cache_configuration(lib, change, word):  # noqa: F811
    for call in (_append, _attend, _keep):
        _refused(lib, call(lib, _cfg(**change)), CONFIG, word)
    n = C.c_size_t(0)
    _refused(lib, lib.sprinter_cache_attend_bytes(_cfg(**change), 4, 3, 4, 5, C.byref(n)), CONFIG, word)


def test_what_all_calls_on_a_cache_refuse(lib):  # noqa: F811
    for call in (_append, _attend, _keep):
        for name in ("keys", "values", "table"):
            _refused(lib, call(lib, **{name: None}), NULL, "NULL array")
        for name in ("keys", "values"):
            _refused(lib, call(lib, **{name: A + 8}), RANGE, "16-byte")
        _refused(lib, call(lib, table=A + 2), RANGE, "table")
        _refused(lib, call(lib, ldt=3), RANGE, "pages")
        _refused(lib, call(lib, n_seq=-1), RANGE, "sequences")
        _refused(lib, call(lib, n_seq=(1 << 20) + 1), RANGE, "sequences")
        _refused(lib, call(lib, n_table=-1), RANGE, "slots")
        _refused(lib, call(lib, n_table=1 << 26, ldt=1 << 26), RANGE, "slots")
        assert call(lib, n_seq=0) == 0
    for call in (_append, _attend):
        for layer in (-1, 2):
            _refused(lib, call(lib, layer=layer), RANGE, "layer")
        _refused(lib, call(lib, T=-1), RANGE, "rows")
        _refused(lib, call(lib, T=(1 << 20) + 1), RANGE, "rows")
        for H in (3, 5, -2, 4098):
            _refused(lib, call(lib, H=H), RANGE, "n_head")
        assert call(lib, T=0) == 0
    for name, layout, good in (("append", ops._APPEND, APPEND), ("attend", ops._ATTEND, ATTEND), ("keep", ops._KEEP, KEEP)):
        call = getattr(lib, "sprinter_cache_" + name)
        _refused(lib, call(None, _packed(layout, good, {}), None), NULL, "configuration")
        _refused(lib, call(_cfg(), None, None), NULL, "arguments")


def test_append_arguments(lib):  # noqa: F811
    for name in ("seq", "slot", "freq", "k", "v", "q", "qo"):
        _refused(lib, _append(lib, **{name: None}), NULL, "NULL array")
    for n in (-2, 63, 66):
        _refused(lib, _append(lib, n=n), RANGE, "n_turned")
    _refused(lib, _append(lib, pairs=2), CONFIG, "pairs")
    _refused(lib, _append(lib, type=2), CONFIG, "rows_dtype")
    for name in ("ldk", "ldv"):
        _refused(lib, _append(lib, **{name: 127}), RANGE, "closer")
    for name in ("ldq", "ldqo"):
        _refused(lib, _append(lib, **{name: 255}), RANGE, "closer")
    for name, by in (("seq", 2), ("slot", 1), ("pos", A + 2), ("freq", 4), ("k", 1), ("v", 1), ("q", 1), ("qo", 1)):
        _refused(lib, _append(lib, **{name: by if by > A else A + by}), RANGE, "aligned")
    _refused(lib, _append(lib, type=0, k=A + 2), RANGE, "aligned")


def test_attend_arguments(lib):  # noqa: F811
    for name in ("lens", "first", "q", "y"):
        _refused(lib, _attend(lib, **{name: None}), NULL, "NULL array")
    for words in (0, 17, -1):
        _refused(lib, _attend(lib, words=words), RANGE, "n_words")
    for scale in (float("nan"), float("inf"), 3e38):
        _refused(lib, _attend(lib, scale=scale), CONFIG, "scale")
    for name in ("ldq", "ldy"):
        _refused(lib, _attend(lib, **{name: 248}), RANGE, "closer")
        _refused(lib, _attend(lib, **{name: 260}), RANGE, "16-byte")
    for name in ("q", "y"):
        _refused(lib, _attend(lib, **{name: A + 8}), RANGE, "16-byte")
    _refused(lib, _attend(lib, T=1 << 20, H=16, ldq=1024, ldy=1024), RANGE, "2^23")
    for name, by in (("lens", 2), ("first", 2), ("vis", 4)):
        _refused(lib, _attend(lib, **{name: A + by}), RANGE, "aligned")
    _refused(lib, _attend(lib, work=A + 128), WORKSPACE, "256-byte")
    n = C.c_size_t(0)
    assert lib.sprinter_cache_attend_bytes(_cfg(), 4, 3, 400, 5, C.byref(n)) == 0
    if n.value:
        _refused(lib, _attend(lib, n_table=400, ldt=400, bytes=n.value - 1), WORKSPACE, "needed")
        _refused(lib, _attend(lib, n_table=400, ldt=400, work=None), NULL, "workspace")
    _refused(lib, lib.sprinter_cache_attend_bytes(_cfg(), 4, 3, 4, 5, None), NULL, "result")
    _refused(lib, lib.sprinter_cache_attend_bytes(_cfg(), 3, 3, 4, 5, C.byref(n)), RANGE, "n_head")


def test_keep_arguments(lib):  # noqa: F811
    for name in ("lens", "first", "path", "n_keep"):
        _refused(lib, _keep(lib, **{name: None}), NULL, "NULL array")
        _refused(lib, _keep(lib, **{name: A + 2}), RANGE, "aligned")
    _refused(lib, _keep(lib, n_path=-1), RANGE, "path")
    _refused(lib, _keep(lib, ldp=3), RANGE, "path")
    assert _keep(lib, n_path=0) == 0


def test_logits_arguments(lib):  # noqa: F811
    _refused(lib, lib.sprinter_adjust_logits(None, None), NULL, "arguments")
    for change, code, word in ((dict(dtype=2), CONFIG, "dtype"), (dict(vocab=0), CONFIG, "vocab"), (dict(vocab=(1 << 24) + 1), CONFIG, "vocab"),
                               (dict(n_rows=-1), RANGE, "rows"), (dict(n_rows=(1 << 20) + 1), RANGE, "rows"), (dict(n_rows=(1 << 19) + 1), RANGE, "draft"),
                               (dict(n_seq=-1), RANGE, "sequences"), (dict(n_tokens=-1), RANGE, "n_tokens"), (dict(n_tokens=(1 << 19) + 1), RANGE, "n_tokens"),
                               (dict(n_words=0), RANGE, "n_words"), (dict(n_words=17), RANGE, "n_words"), (dict(n_bias=2048), RANGE, "n_bias"),
                               (dict(n_bias=-1), RANGE, "n_bias"), (dict(n_mask=-1), RANGE, "masks"), (dict(logits=None), NULL, "logits"), (dict(out=None), NULL, "out"),
                               (dict(bias=None), NULL, "together"), (dict(bias_ids=None), NULL, "together"), (dict(tokens=None), NULL, "without tokens"),
                               (dict(tokens=None, n_token=None), NULL, "without tokens"), (dict(mask=None), NULL, "without mask"),
                               (dict(first=None, n_seq=2), RANGE, "without first"), (dict(mask_row=None), RANGE, "without mask_row"),
                               (dict(ld_logits=99), RANGE, "closer"), (dict(ld_out=99), RANGE, "closer"), (dict(ld_tokens=49), RANGE, "closer"),
                               (dict(ld_bias=7), RANGE, "closer"), (dict(ld_bias_ids=7), RANGE, "closer"), (dict(ld_mask=3), RANGE, "closer")):
        _refused(lib, _logits(lib, **change), code, word)
    for name in ("logits", "out", "first", "tokens", "n_token", "n_prompt", "repetition", "presence", "frequency", "draft", "visible", "bias_ids", "bias", "mask",
                 "mask_row"):
        _refused(lib, _logits(lib, **{name: A + (4 if name == "visible" else 2)}), RANGE, "aligned")
    half = 1 << 19                                       # each is a limit that is allowed; together a token's count would be 2^20
    _refused(lib, _logits(lib, n_rows=half, n_tokens=half, ld_tokens=half), RANGE, "together")
    assert _logits(lib, n_rows=0) == 0


# ------------------------------------------------------------------------------------------- the torch entry points, without a device
I = torch.int32  # noqa: E741
f = torch.ones


def z(*s):
    return torch.zeros(*s, dtype=I)


def _cache(dtype=torch.float32):
    return ops.PagedCache(torch.zeros(2, 10, 2, 16, 64, dtype=dtype), torch.zeros(2, 10, 2, 16, 64, dtype=dtype))


GOOD = dict(append=lambda c, **kw: c.append(**{**dict(layer=0, keys=f(5, 128), values=f(5, 128), table=z(3, 4), seq=z(5), slot=z(5), q=f(5, 256),
                                                      freq=torch.ones(32, dtype=torch.float64)), **kw}),
            attend=lambda c, **kw: c.attend(**{**dict(layer=0, q=f(5, 256), table=z(3, 4), lens=z(3), first=z(4), visible=torch.zeros(5, 1, dtype=torch.int64)), **kw}),
            keep=lambda c, **kw: c.keep(**{**dict(table=z(3, 4), lens=z(3), first=z(4), path=z(3, 4), n_keep=z(3)), **kw}),
            logits=lambda c, **kw: ops.adjust_logits(**{**dict(logits=f(5, 100), first=z(4), tokens=z(3, 9), n_token=z(3), n_prompt=z(3), repetition=f(3), presence=f(3),
                                                               frequency=f(3), draft=z(5), visible=torch.zeros(5, 1, dtype=torch.int64), bias_ids=z(3, 2), bias=f(3, 2),
                                                               mask=z(2, 4), mask_row=z(5)), **kw}))


@pytest.mark.parametrize("call, change, word", [
    ("append", dict(keys=f(5, 127)), "keys"), ("append", dict(keys=f(5, 128).double()), "keys"), ("append", dict(values=f(4, 128)), "values"),
    ("append", dict(values=f(5, 128).bfloat16()), "values"), ("append", dict(q=f(5, 250)), "q"), ("append", dict(q=f(4, 256)), "q"), ("append", dict(q=f(5, 0)), "q"),
    ("append", dict(seq=z(4)), "seq"), ("append", dict(slot=z(5).long()), "slot"), ("append", dict(slot=z(10)[::2]), "slot"), ("append", dict(pos=z(6)), "pos"),
    ("append", dict(freq=f(32)), "freq"), ("append", dict(freq=f(2, 16).double()), "freq"), ("append", dict(pairs="both"), "pairs"),
    ("append", dict(q=None, q_out=f(5, 256)), "q_out"), ("append", dict(q_out=f(5, 128)), "q_out"), ("append", dict(q_out=f(5, 256).bfloat16()), "q_out"),
    ("append", dict(layer=2 ** 32), "32 bits"), ("append", dict(layer=0.0), "layer"), ("append", dict(table=z(3, 4).long()), "table"), ("append", dict(table=z(12)), "table"),
    ("append", dict(keys=None), "keys"), ("attend", dict(q=f(5, 250)), "q"), ("attend", dict(q=f(5, 256).bfloat16()), "q"), ("attend", dict(lens=z(4)), "lens"),
    ("attend", dict(first=z(5)), "first"), ("attend", dict(first=z(0)), "first"), ("attend", dict(first=None), "first"),
    ("attend", dict(visible=torch.zeros(5, 0, dtype=torch.int64)), "visible"), ("attend", dict(visible=z(5, 1)), "visible"),
    ("attend", dict(visible=torch.zeros(5, dtype=torch.int64)), "visible"), ("attend", dict(scale=torch.tensor(1.0)), "plain number"), ("attend", dict(scale="1"), "scale"), ("attend", dict(scale=1e39), "float32"), ("logits", dict(presence=torch._efficientzerotensor(3)), "without memory"),
    ("append", dict(pos=torch._efficientzerotensor(5, dtype=I)), "without memory"),
    ("attend", dict(out=f(5, 128)), "out"), ("attend", dict(q=f(256, 5).t()), "adjacent"), ("keep", dict(path=z(2, 4)), "path"), ("keep", dict(n_keep=z(4)), "n_keep"),
    ("keep", dict(first=z(3)), "first"), ("keep", dict(lens=z(3).long()), "lens"), ("logits", dict(logits=f(5, 100).half()), "logits"), ("logits", dict(logits=f(500)), "logits"),
    ("logits", dict(tokens=z(4, 9)), "tokens"), ("logits", dict(n_token=z(4)), "n_token"), ("logits", dict(repetition=f(3).double()), "repetition"),
    ("logits", dict(draft=z(4)), "draft"), ("logits", dict(bias=None), "bias"), ("logits", dict(bias_ids=None), "bias_ids"), ("logits", dict(bias=f(3, 3)), "bias"),
    ("logits", dict(mask=z(2, 3)), "mask"), ("logits", dict(mask_row=z(4)), "mask_row"), ("logits", dict(out=f(5, 99)), "out"), ("logits", dict(mask=z(0, 4), mask_row=None), "no masks"),
    ("logits", dict(presence=1.0), "presence")])
def test_arguments(no_device, lib, call, change, word):  # noqa: F811
    with pytest.raises(ValueError, match=word):
        GOOD[call](_cache(), **change)
    assert not no_device


def test_good_arguments_reach_the_library(no_device, lib):  # noqa: F811
    for call in GOOD.values():
        call(_cache())
    assert no_device == ["sprinter_cache_append", "sprinter_cache_attend", "sprinter_cache_keep", "sprinter_adjust_logits"]
    ops.adjust_logits(f(5, 100), z(4), tokens=z(3, 0), n_token=z(3))          # an empty history, no masks
    ops.adjust_logits(f(5, 100), mask=z(0, 4), mask_row=z(5))


def test_caches_that_are_none(no_device, lib):  # noqa: F811
    for keys, values in ((f(2, 10, 2, 16), f(2, 10, 2, 16)), (f(1, 2, 2, 16, 64).half(),) * 2, (f(1, 2, 2, 16, 64), f(1, 2, 2, 16, 32)),
                         (f(1, 2, 2, 16, 64), f(1, 2, 2, 16, 64).bfloat16()), (f(1, 2, 2, 64, 16).transpose(3, 4), f(1, 2, 2, 16, 64))):
        with pytest.raises(ValueError):
            ops.PagedCache(keys, values)


def test_a_cache_keeps_its_tensors(no_device):  # noqa: F811
    c = _cache()
    for name in ("keys", "values"):
        with pytest.raises(AttributeError):
            setattr(c, name, f(1, 1, 1, 8, 64))


def test_gradients_are_no_matter_where_they_are_off(no_device, lib):  # noqa: F811
    with torch.no_grad():
        GOOD["attend"](_cache(), q=torch.ones(5, 256, requires_grad=True))
        GOOD["logits"](_cache(), logits=torch.ones(5, 100, requires_grad=True), bias=torch.ones(3, 2, requires_grad=True))
    assert len(no_device) == 2


def test_lazy_clones_are_written_apart(no_device, lib):  # noqa: F811
    """A lazy clone shares its memory until one of the two is written: its address is asked for writing."""
    t = f(5, 256)
    u = torch._lazy_clone(t)
    GOOD["attend"](_cache(), out=u)
    assert u.data_ptr() != t.data_ptr()


def test_gradients_and_tangents_are_refused(no_device, lib):  # noqa: F811
    import torch.autograd.forward_ad as fwd
    c = _cache()
    grad = lambda *s: torch.ones(*s, requires_grad=True)  # noqa: E731
    for call, name, shape in (("append", "keys", (5, 128)), ("append", "values", (5, 128)), ("append", "q", (5, 256)), ("attend", "q", (5, 256)), ("logits", "logits", (5, 100)),
                              ("logits", "bias", (3, 2)), ("logits", "repetition", (3,))):
        with pytest.raises(ValueError, match="gradients"):
            GOOD[call](c, **{name: grad(*shape)})
        with fwd.dual_level(), pytest.raises(ValueError, match="tangents"):
            GOOD[call](c, **{name: fwd.make_dual(f(*shape), f(*shape))})
    with pytest.raises(ValueError, match="gradients"):
        ops.PagedCache(grad(2, 10, 2, 16, 64), f(2, 10, 2, 16, 64))
    assert not no_device


def test_tensors_written_in_place_are_known_to_autograd(no_device, lib):  # noqa: F811
    c = _cache()
    GOOD["append"](c)
    GOOD["keep"](c)
    GOOD["attend"](c)
    assert c.keys._version == c.values._version == 2
    for call, name, t in (("append", "q_out", f(5, 256)), ("attend", "out", f(5, 256)), ("logits", "out", f(5, 100))):
        assert GOOD[call](_cache(), **{name: t}) is t and t._version == 1
    with torch.inference_mode():
        c = _cache()
        GOOD["append"](c)
        GOOD["logits"](c, out=f(5, 100))


def _shrunk(t, left):
    """`t` after its storage was cut to `left` bytes, as programs do that free a tensor's memory and keep the tensor."""
    t.untyped_storage().resize_(left)
    return t


WITHOUT = dict(append=dict(keys=lambda: f(5, 128), values=lambda: f(5, 128), table=lambda: z(3, 4), seq=lambda: z(5), slot=lambda: z(5), q=lambda: f(5, 256), pos=lambda: z(5),
                           freq=lambda: torch.ones(32, dtype=torch.float64), q_out=lambda: f(5, 256)),
               attend=dict(q=lambda: f(5, 256), table=lambda: z(3, 4), lens=lambda: z(3), first=lambda: z(4), visible=lambda: torch.zeros(5, 1, dtype=torch.int64),
                           out=lambda: f(5, 256)),
               keep=dict(table=lambda: z(3, 4), lens=lambda: z(3), first=lambda: z(4), path=lambda: z(3, 4), n_keep=lambda: z(3)),
               logits=dict(logits=lambda: f(5, 100), first=lambda: z(4), tokens=lambda: z(3, 9), n_token=lambda: z(3), n_prompt=lambda: z(3), repetition=lambda: f(3),
                           presence=lambda: f(3), frequency=lambda: f(3), draft=lambda: z(5), visible=lambda: torch.zeros(5, 1, dtype=torch.int64), bias_ids=lambda: z(3, 2),
                           bias=lambda: f(3, 2), mask=lambda: z(2, 4), mask_row=lambda: z(5), out=lambda: f(5, 100)))


@pytest.mark.parametrize("call, name", [(c, n) for c, names in WITHOUT.items() for n in names])
def test_tensors_whose_memory_was_freed(no_device, lib, call, name):  # noqa: F811
    """All of it, the last byte of it, and a view's that begins behind it: none is taken for an array that is not given."""
    make = WITHOUT[call][name]
    whole = make()
    behind = torch.cat([whole, make()])[whole.shape[0]:]
    for t, left in ((whole, 0), (make(), whole.numel() * whole.element_size() - 1), (behind, 0), (torch.cat([make(), make()])[whole.shape[0]:], whole.numel() * whole.element_size())):
        t = _shrunk(t, left)
        with pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
            GOOD[call](_cache(), **{name: t})
        with torch.no_grad(), pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
            GOOD[call](_cache(), **{name: t})
    with pytest.raises(ValueError, match="mask: a tensor without memory"):
        ops.adjust_logits(f(2, 100), mask=_shrunk(z(2, 4), 0))
    assert not no_device


@pytest.mark.parametrize("name", ["keys", "values"])
def test_caches_whose_memory_was_freed(no_device, lib, name):  # noqa: F811
    """Before the object is made, or afterwards: neither its address nor its sizes are kept."""
    shape = (2, 10, 2, 16, 64)
    good = {"keys": f(*shape), "values": f(*shape)}
    with pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
        ops.PagedCache(**{**good, name: _shrunk(f(*shape), 0)})
    for left in (0, 2 * 10 * 2 * 16 * 64 * 4 - 1):
        for both in (f(*shape), f(2, *shape)[1]):
            cache = ops.PagedCache(**{**good, name: both})
            _shrunk(both, left)
            for call in ("append", "attend", "keep"):
                with pytest.raises(ValueError, match=f"{name}: a tensor without memory"):
                    GOOD[call](cache)
    t = f(*shape)
    cache = ops.PagedCache(**{**good, name: t})
    t.resize_(1, 10, 2, 16, 64)
    for call in ("append", "attend", "keep"):
        with pytest.raises(ValueError, match=f"{name}: "):
            GOOD[call](cache)
    assert not no_device
