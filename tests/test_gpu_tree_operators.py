"""The operators of a round of drafted trees over a cache in pages, against their definitions in float64."""
import numpy as np
import pytest
import torch
import tree_math as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INF, NAN = float("inf"), float("nan")


def _ops():
    from paper_2502_04557_amd import operators
    return operators


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Batch:
    """A cache with random contents, a table of shuffled pages and a batch of trees."""

    def __init__(self, seed, dtype, lens, nodes, H, KVH, dh, page, layers=1, spare=2, wide=0, only_cache=False):
        self.g = torch.Generator().manual_seed(seed)
        self.lens_, self.nodes_, self.H, self.KVH, self.dh, self.page, self.dtype = lens, nodes, H, KVH, dh, page, TYPES[dtype]
        need = [-(-(l + n) // page) for l, n in zip(lens, nodes)]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=self.g).to(torch.int32)
        table = torch.full((len(lens), max(max(need), 1) + wide), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table.to(DEV)
        shape = (layers, pages, KVH, page, dh)
        self.keys, self.values = self.normal(*shape).to(self.dtype), self.normal(*shape).to(self.dtype)
        self.cache = _ops().PagedCache(self.keys, self.values)
        self.lens, self.first = _ints(lens), _ints(np.concatenate([[0], np.cumsum(nodes)]).tolist())
        self.T = sum(nodes)
        self.q = self.normal(self.T, H * dh).to(self.dtype)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g).to(DEV)

    def seen(self, share=0.5, words=None):
        """A random half of all nodes for every row, itself or not."""
        words = words or max(1, -(-max(self.nodes_) // 64))
        bits = torch.rand(self.T, words, 64, generator=self.g) < share
        return (bits.long() << torch.arange(64)).sum(2).to(DEV)

    def check(self, y=None, visible=None, layer=0, scale=None, q=None):
        q = self.q if q is None else q
        if y is None:
            y = self.cache.attend(layer, q, self.table, self.lens, self.first, visible=visible, scale=scale)
        half = self.dtype == torch.bfloat16
        want, bound, mine = M.attend(self.keys[layer], self.values[layer], self.table, self.lens, self.first, visible, q.reshape(self.T, self.H, self.dh),
                                     self.dh ** -0.5 if scale is None else scale, half)
        got = y.double().cpu().reshape(self.T, self.H, self.dh)
        off = (got - want).abs()[mine]
        bad = ~(off <= bound[mine])
        assert not bad.any(), (int(bad.sum()), off[bad][:4], bound[mine][bad][:4], torch.nonzero(bad)[:4])
        # rounding alone leaves far less than the bound in the mean: a key, a block or a column that is wrong does not
        if mine.any() and half:
            norm = want[mine].norm()
            assert (got - want)[mine].norm() <= 2.0 ** -8 * norm + 1e-30
        return y


# ----------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("dh, H, KVH, page, turned, T, off", [
    (64, 4, 4, 8, 64, 1, 0), (128, 8, 2, 16, 128, 7, 0), (64, 25, 25, 32, 32, 5, 0), (128, 6, 1, 1024, 30, 33, 0), (64, 3, 3, 64, 2, 9, 1), (128, 5, 5, 128, 126, 130, 4),
    (128, 32, 8, 16, 128, 300, 0), (64, 7, 7, 8, 48, 67, 8), (64, 0, 2, 16, 64, 11, 0), (64, 2, 2, 16, 0, 19, 0)])
def test_append(dtype, rows, pairs, dh, H, KVH, page, turned, T, off):
    g = torch.Generator().manual_seed(T + dh + turned)
    B, layers = 5, 3
    n_table = -(-(T + 40) // page)
    pages = B * n_table + 3
    keys = torch.randn(layers, pages, KVH, page, dh, generator=g).to(TYPES[dtype])
    values = torch.randn(layers, pages, KVH, page, dh, generator=g).to(TYPES[dtype])
    table = torch.randperm(pages, generator=g)[:B * n_table].to(torch.int32).reshape(B, n_table)
    table[3, 0] = -1                                      # a sequence whose first page is not there, one that points beyond the cache
    table[4, -1] = pages
    seq = torch.randint(-1, B + 1, (T,), generator=g).to(torch.int32)
    slot = torch.zeros(T, dtype=torch.int32)
    nth = [0] * (B + 2)
    for t in range(T):                                    # every (sequence, slot) once, slots beyond the table among them
        slot[t] = nth[seq[t]] * 37 % (n_table * page + 3)
        nth[seq[t]] += 1
    used, unique = set(), []
    for t in range(T):
        k = (int(seq[t]), int(slot[t]))
        unique.append(k not in used)
        used.add(k)
    seq[~torch.tensor(unique)] = -1
    if T > 4:
        slot[2] = -5
    pos = torch.randint(0, 200000, (T,), generator=g).to(torch.int32)
    freq = 5e5 ** (-torch.arange(0, turned, 2, dtype=torch.float64) / max(turned, 1))
    w = (H + 2 * KVH) * dh + off
    qkv = torch.randn(T, w + off, generator=g).to(TYPES[rows])[:, off:]
    q, k, v = qkv[:, :H * dh], qkv[:, H * dh:(H + KVH) * dh], qkv[:, (H + KVH) * dh:(H + 2 * KVH) * dh]
    K, V = keys.to(DEV), values.to(DEV)
    cache = _ops().PagedCache(K, V)
    dq = qkv.to(DEV)
    args = (dq[:, H * dh:(H + KVH) * dh], dq[:, (H + KVH) * dh:(H + 2 * KVH) * dh], table.to(DEV), seq.to(DEV), slot.to(DEV))
    q_out = torch.full((T, H * dh), 7.0, dtype=TYPES[dtype], device=DEV) if H else None
    got = cache.append(1, *args, q=dq[:, :H * dh] if H else None, pos=pos.to(DEV), freq=freq.to(DEV) if turned else None, pairs=pairs, q_out=q_out)
    assert got is q_out
    half = dtype == "bf16"
    yk, bk = M.turned(k.double().numpy().reshape(T, KVH, dh), pos.numpy(), freq.numpy(), pairs, half)
    yv = v.double().numpy().reshape(T, KVH, dh)
    wk, wv, ek = keys.double().numpy(), values.double().numpy(), np.zeros(keys.shape)
    for t in range(T):
        at = M.slot_of(table.numpy(), pages, page, int(seq[t]), int(slot[t])) if 0 <= seq[t] < B else None
        if at:
            wk[1, at[0], :, at[1]], ek[1, at[0], :, at[1]] = yk[t], bk[t]
            wv[1, at[0], :, at[1]] = torch.from_numpy(yv[t]).to(TYPES[dtype]).double().numpy()      # rounded once
    assert (np.abs(K.double().cpu().numpy() - wk) <= ek).all()
    assert np.array_equal(V.double().cpu().numpy(), wv)
    if H:
        yq, bq = M.turned(q.double().numpy().reshape(T, H, dh), pos.numpy(), freq.numpy(), pairs, half)
        there = ((seq >= 0) & (seq < B)).numpy()
        out = got.double().cpu().numpy().reshape(T, H, dh)
        assert (np.abs(out - yq) <= bq)[there].all()
        assert (out[~there] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_append_turns_queries_in_place_and_takes_the_slot_as_position(dtype, pairs):
    b = Batch(5, dtype, [30, 11], [9, 4], 6, 2, 64, 16)
    seq, slot = _ints([0] * 9 + [1] * 4), _ints(list(range(30, 39)) + list(range(11, 15)))
    freq = 1e4 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device=DEV) / 64)
    k, v = b.normal(13, 128).to(b.dtype), b.normal(13, 128).to(b.dtype)
    q = b.q.clone()
    want = b.cache.append(0, k, v, b.table, seq, slot, q=q, freq=freq, pairs=pairs)
    keys = b.keys.clone()
    assert torch.equal(q, b.q)
    again = b.cache.append(0, k, v, b.table, seq, slot, q=q, pos=slot.clone(), freq=freq, pairs=pairs, q_out=q)
    assert again is q and torch.equal(q, want) and torch.equal(b.keys, keys)


def test_append_at_far_and_broken_positions():
    """Positions up to 31 bits; a frequency that is not finite reaches its own columns only."""
    b = Batch(6, "f32", [40], [4], 2, 2, 64, 8)
    pos = _ints([2 ** 31 - 1, 2 ** 24 + 1, 123456789, -7])
    freq = 5e5 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device=DEV) / 64)
    k = b.normal(4, 128)
    q = b.cache.append(0, k, k, b.table, _ints([0] * 4), _ints([40, 41, 42, 43]), q=k, pos=pos, freq=freq)
    y, e = M.turned(k.double().cpu().numpy().reshape(4, 2, 64), pos.cpu().numpy(), freq.cpu().numpy(), "halves", False)
    assert (np.abs(q.double().cpu().numpy().reshape(4, 2, 64) - y) <= e).all()
    freq[3] = INF
    bad = b.cache.append(0, k, k, b.table, _ints([0] * 4), _ints([40, 41, 42, 43]), q=k, pos=pos, freq=freq).reshape(4, 2, 64)
    hit = torch.zeros(64, dtype=torch.bool, device=DEV)
    hit[[3, 35]] = True
    assert bad[..., hit].isnan().all() and torch.equal(bad[..., ~hit], q.reshape(4, 2, 64)[..., ~hit])


# ----------------------------------------------------------------------------------------------------------------- attend
SHAPES = [([0], [1], 1, 1, 64, 8), ([5], [1], 4, 1, 128, 16), ([31, 32, 33, 0, 1], [1, 1, 1, 1, 1], 8, 8, 64, 8), ([100, 7, 64], [3, 16, 17], 8, 2, 128, 32),
          ([0, 3, 250], [33, 64, 1], 25, 25, 64, 16), ([129, 500], [40, 5], 12, 4, 64, 64), ([700, 20, 0, 95], [9, 0, 31, 2], 6, 2, 128, 128),
          ([1030], [1], 32, 8, 128, 16), ([63, 255, 511, 1000, 12, 300], [8, 7, 6, 5, 4, 3], 10, 2, 128, 16), ([2000], [64], 16, 2, 64, 1024), ([90], [20], 40, 1, 64, 16),
          ([37] * 20, [2] * 20, 5, 5, 128, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh, page", SHAPES)
def test_attend(dtype, lens, nodes, H, KVH, dh, page):
    b = Batch(sum(lens) + H, dtype, lens, nodes, H, KVH, dh, page)
    b.check()                                             # chains
    b.check(visible=b.seen())                             # any subset, rows without anything among them
    b.check(visible=torch.zeros(b.T, 1, dtype=torch.int64, device=DEV), scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh, words", [([40, 0], [70, 129], 4, 2, 64, 3), ([9], [300], 2, 1, 128, 5), ([200], [200], 8, 1, 64, 2), ([3], [1000], 1, 1, 64, 16)])
def test_attend_many_nodes(dtype, lens, nodes, H, KVH, dh, words):
    """Several words of a mask, nodes behind the last word, chains of a piece of a prompt."""
    b = Batch(words, dtype, lens, nodes, H, KVH, dh, 16)
    b.check()
    b.check(visible=b.seen(0.3, words))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, H, KVH, dh", [([9000, 40, 2500, 1], [5, 3, 20, 1], 8, 2, 128), ([5000], [1], 4, 4, 64), ([70, 6000, 0], [64, 2, 9], 16, 4, 64)])
def test_attend_long_and_uneven(dtype, lens, nodes, H, KVH, dh):
    b = Batch(9, dtype, lens, nodes, H, KVH, dh, 32)
    b.check(visible=b.seen())
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_peaks_and_ties(dtype):
    """Scores that grow along the context, one that towers over the rest, all alike; scores far below 0."""
    b = Batch(3, dtype, [300, 77], [4, 9], 4, 2, 64, 16)
    for s in (0.0, 3.0, -3.0):
        b.check(scale=s)
    b.keys[0, b.table[0, 250 // 16].long(), :, 250 % 16] = 6 * b.q[0, :64]
    b.check()
    b.keys[:] = -b.keys[:].abs() * 20
    b.q[:] = b.q.abs() * 20
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_attend_strides_layers_and_rows_of_no_sequence(dtype, dh):
    b = Batch(4, dtype, [50, 3, 20], [6, 2, 5], 4, 2, dh, 8, layers=3, wide=3)
    wide = b.normal(b.T + 7, 4 * dh * 3).to(b.dtype)
    q = wide[3:3 + b.T, 4 * dh:8 * dh]
    vis = b.seen()
    for layer in (0, 2):
        b.check(visible=vis, layer=layer, q=q)
    want = b.cache.attend(1, q, b.table, b.lens, b.first, visible=vis)
    out = torch.full((b.T + 7, 4 * dh * 2), 5.0, dtype=b.dtype, device=DEV)
    # rows in front of the first sequence and behind the last one, a gap in no place of `first`; a table of a wider array
    rows = wide[:, 4 * dh:8 * dh]
    table = torch.full((3, 40), 99, dtype=torch.int32, device=DEV)
    table[:, 10:10 + b.table.shape[1]] = b.table
    more = torch.zeros(b.T + 7, 1, dtype=torch.int64, device=DEV)
    more[3:3 + b.T] = vis
    got = b.cache.attend(1, rows, table[:, 10:10 + b.table.shape[1]], b.lens, b.first + 3, visible=more, out=out[:, :4 * dh])
    assert got.data_ptr() == out.data_ptr() and torch.equal(got[3:3 + b.T], want)
    assert (out[:3] == 5).all() and (out[3 + b.T:] == 5).all() and (out[:, 4 * dh:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_pages_that_are_not_there(dtype):
    """Entries outside the cache, and lengths beyond the table: those slots are not seen."""
    b = Batch(8, dtype, [100, 45, 64], [5, 8, 1], 4, 2, 64, 8)
    b.table[0, 3], b.table[0, 12], b.table[1, :] = -1, b.keys.shape[1], -7
    b.check()
    b.check(visible=b.seen())
    y = b.cache.attend(0, b.q, b.table, b.lens, b.first)
    assert (y[5:13] == 0).all()                           # a sequence without any page
    b.lens[2] = 4000
    b.check(visible=b.seen(1.0))
    b.lens[2] = -3
    z = b.cache.attend(0, b.q, b.table, b.lens, b.first)
    assert torch.equal(z[:13], y[:13]) and z.isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh, H, KVH, nodes, page", [(64, 4, 2, 12, 8), (128, 8, 1, 40, 16), (128, 2, 2, 1, 64), (64, 16, 2, 64, 32)])
@pytest.mark.parametrize("what", [NAN, INF, -INF])
def test_attend_what_is_not_seen_does_not_reach(dtype, dh, H, KVH, nodes, page, what):
    """Values that are not finite in slots behind the last node, in unused pages and in nodes that a row does not see."""
    lens, n = [70, 33], [nodes, max(1, nodes - 1)]
    b = Batch(11, dtype, lens, n, H, KVH, dh, page)
    vis = b.seen()
    sick = 2 % min(n)                                     # node `sick` of each sequence is seen by odd rows alone
    odd = torch.tensor([(t - f) % 2 for f, c in zip((0, n[0]), n) for t in range(f, f + c)], device=DEV)
    vis = torch.where(odd[:, None] == 1, vis | (1 << sick), vis & ~(1 << sick))
    want = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis)
    used = torch.zeros(b.keys.shape[1], page, dtype=torch.bool)
    for s, (l, c) in enumerate(zip(lens, n)):
        for i in range(l + c):
            p = M.slot_of(b.table.cpu().numpy(), b.keys.shape[1], page, s, i)
            used[p] = True
    unused = ~used.to(DEV)[None, :, None, :, None].expand_as(b.keys)
    for t in (b.keys, b.values):
        t[unused] = what
    assert torch.equal(b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis), want)
    before = b.keys.clone(), b.values.clone()
    for s, l in enumerate(lens):
        p = M.slot_of(b.table.cpu().numpy(), b.keys.shape[1], page, s, l + sick)
        b.values[0, p[0], :, p[1], 3:9] = what
    got = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis)
    assert torch.equal(got[odd == 0], want[odd == 0])
    y = got[odd == 1].reshape(-1, H, dh)
    keep = torch.ones(dh, dtype=torch.bool, device=DEV)
    keep[3:9] = False
    assert torch.equal(y[..., keep], want[odd == 1].reshape(-1, H, dh)[..., keep])
    hit = y[..., 3:9]
    assert (hit.isnan() if what != what else hit == what).all()
    b.keys.copy_(before[0])
    b.values.copy_(before[1])
    for s, l in enumerate(lens):
        p = M.slot_of(b.table.cpu().numpy(), b.keys.shape[1], page, s, l + sick)
        b.keys[0, p[0], :, p[1]] = NAN
    got = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis)
    assert torch.equal(got[odd == 0], want[odd == 0]) and got[odd == 1].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_broken_queries_and_scores(dtype):
    """A query that is not finite makes its own row NaN; scores of -infinity have no weight, a row of them alone gives zeros."""
    b = Batch(12, dtype, [50], [6], 4, 2, 64, 16)
    want = b.cache.attend(0, b.q, b.table, b.lens, b.first)
    q = b.q.clone()
    q[2, :64] = NAN
    got = b.cache.attend(0, q, b.table, b.lens, b.first)
    assert got[2, :64].isnan().all()
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[2, :64] = False
    assert torch.equal(got[rest], want[rest])
    b.q[:] = b.q.abs() + 0.1
    at = b.table[0, 0].long()
    b.keys[0, at, :, 5] = -INF                            # one committed key: no weight
    y = b.cache.attend(0, b.q, b.table, b.lens, b.first)
    b.keys[0, at, :, 5] = 0
    b.table[0, 0], kept = -1, int(at)
    b.keys[:] = -INF
    assert (b.cache.attend(0, b.q, b.table, b.lens, b.first) == 0).all()
    assert y.isfinite().all() and kept >= 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_offsets_beyond_32_bits(dtype):
    """Pages at the end of a cache of more than 2^32 bytes and 2^31 elements per array, and a layer behind it."""
    page, KVH, dh = 128, 8, 128
    pages = 2 ** 31 // (page * KVH * dh) + 40
    keys = torch.empty(2, pages, KVH, page, dh, dtype=TYPES[dtype], device=DEV)
    values = torch.empty_like(keys)
    b = Batch(13, dtype, [300, 90], [5, 12], 16, KVH, dh, page)
    n = b.keys.shape[1]
    keys[1, -n:], values[1, -n:] = b.keys[0], b.values[0]
    table = torch.where(b.table >= 0, b.table + (pages - n), b.table)
    cache = _ops().PagedCache(keys, values)
    vis = b.seen()
    want = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis)
    assert torch.equal(cache.attend(1, b.q, table, b.lens, b.first, visible=vis), want)
    k, v, seq, slot = b.normal(3, KVH * dh), b.normal(3, KVH * dh), _ints([0, 1, 1]), _ints([299, 5, 101])
    cache.append(1, k, v, table, seq, slot)
    b.cache.append(0, k, v, b.table, seq, slot)
    path, n_keep = _ints([[1, 3, 4], [0, 5, 11]]), _ints([3, 3])
    cache.keep(table, b.lens, b.first, path, n_keep)
    b.cache.keep(b.table, b.lens, b.first, path, n_keep)
    assert torch.equal(keys[1, -n:], b.keys[0]) and torch.equal(values[1, -n:], b.values[0])


# ------------------------------------------------------------------------------------------------------------------- keep
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, nodes, KVH, dh, page, layers", [([3], [1], 1, 64, 8, 1), ([20, 0, 61], [15, 9, 40], 3, 64, 16, 4), ([7, 100], [64, 33], 8, 128, 8, 2),
                                                                ([31] * 9, [12] * 9, 25, 64, 32, 3)])
def test_keep(dtype, lens, nodes, KVH, dh, page, layers):
    b = Batch(21, dtype, lens, nodes, KVH, KVH, dh, page, layers=layers)
    g = np.random.default_rng(sum(lens))
    n = max(nodes) + 2
    path, kept = np.full((len(lens), n), -1, np.int32), np.zeros(len(lens), np.int32)
    for s, c in enumerate(nodes):
        kept[s] = g.integers(0, c + 1)
        path[s, :kept[s]] = np.sort(g.choice(c, kept[s], replace=False))
    keys, values = b.keys.double().cpu().numpy(), b.values.double().cpu().numpy()
    args = (b.table.cpu().numpy(), lens, [0, *np.cumsum(nodes)])
    b.cache.keep(b.table, b.lens, b.first, torch.from_numpy(path).to(DEV), torch.from_numpy(kept).to(DEV))
    assert np.array_equal(b.keys.double().cpu().numpy(), M.keep(keys, *args, path, kept))
    assert np.array_equal(b.values.double().cpu().numpy(), M.keep(values, *args, path, kept))


def test_keep_what_moves_nothing():
    """Entries below their place or behind the tree, counts beyond the path, below 0, pages that are not there; bits of NaN move too."""
    b = Batch(22, "bf16", [10, 20, 5, 30], [6, 6, 6, 6], 2, 2, 64, 8)
    b.keys.view(torch.int16)[0, 0] = 0x7fa5
    b.table[3, 30 // 8 + 1] = -1
    path = np.array([[0, 0, 5, 9], [3, 1, 7, -1], [2, 3, 4, 5], [1, 2, 4, 5]], np.int32)
    kept = np.array([4, 4, -2, 9], np.int32)
    lens, first, table = [10, 20, 5, 30], [0, 6, 12, 18, 24], b.table.cpu().numpy()
    want = [M.keep(t.view(torch.int16).cpu().numpy(), table, lens, first, path, kept) for t in (b.keys, b.values)]
    b.cache.keep(b.table, b.lens, b.first, torch.from_numpy(path).to(DEV), torch.from_numpy(kept).to(DEV))
    for t, w in zip((b.keys, b.values), want):
        assert np.array_equal(t.view(torch.int16).cpu().numpy(), w)


# ----------------------------------------------------------------------------------------------------------------- logits
def _logits_case(seed, dtype, B, nodes, V, L, n_bias, words=1):
    g = np.random.default_rng(seed)
    T = sum(nodes)
    first = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    logits = torch.from_numpy((g.standard_normal((T, V)) * 3).astype(np.float32)).to(TYPES[dtype])
    hot = g.integers(-2, V + 2, 12).astype(np.int32)      # ids that come again and again, some outside the vocabulary
    pick = lambda *s: np.where(g.random(s) < 0.5, hot[g.integers(0, 12, s)], g.integers(0, V, s)).astype(np.int32)  # noqa: E731
    kw = dict(tokens=pick(B, L), n_token=g.integers(0, L + 1, B).astype(np.int32), n_prompt=g.integers(0, L + 1, B).astype(np.int32),
              repetition=(0.8 + g.random(B)).astype(np.float32), presence=g.standard_normal(B).astype(np.float32), frequency=g.standard_normal(B).astype(np.float32),
              draft=pick(T), visible=g.integers(0, 2 ** 63, (T, words)).astype(np.int64), bias_ids=pick(B, n_bias), bias=g.standard_normal((B, n_bias)).astype(np.float32),
              mask=g.integers(-2 ** 31, 2 ** 31, (3, (V + 31) // 32)).astype(np.int32), mask_row=g.integers(-1, 4, T).astype(np.int32))
    return logits, first, kw


def _check_logits(logits, first, kw, half, **more):
    dev = {k: None if v is None else torch.from_numpy(v).to(DEV) for k, v in kw.items()}
    got = _ops().adjust_logits(logits.to(DEV), None if first is None else torch.from_numpy(first).to(DEV), **dev, **more)
    want, bound = M.adjust(logits.double().cpu().numpy(), first, kw, half)
    g = got.double().cpu().numpy()
    same = np.isinf(want) | np.isnan(want)
    assert np.array_equal(g[same], want[same], equal_nan=True)
    assert (np.abs(g[~same] - want[~same]) <= bound[~same]).all()
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes, V, L, n_bias", [([1], 1, 1, 1), ([1, 1], 31, 9, 3), ([3, 0, 5], 100, 200, 40), ([1, 9], 4097, 33, 2047), ([2, 2, 2, 1], 50257, 300, 17),
                                                 ([16, 1], 9001, 5000, 8), ([70], 517, 64, 5)])
def test_logits(dtype, nodes, V, L, n_bias):
    logits, first, kw = _logits_case(V, dtype, len(nodes), nodes, V, L, n_bias)
    half = dtype == "bf16"
    _check_logits(logits, first, kw, half)
    off = dict.fromkeys(kw)
    for names in (("tokens", "repetition"), ("tokens", "n_token", "frequency", "presence"), ("draft", "visible", "repetition", "frequency"), ("draft", "presence"),
                  ("bias_ids", "bias"), ("mask", "mask_row"), (), ("tokens", "n_prompt", "repetition", "presence", "bias_ids", "bias")):
        _check_logits(logits, first, {**off, **{n: kw[n] for n in names}}, half)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_without_trees_and_with_many_nodes(dtype):
    half = dtype == "bf16"
    logits, _, kw = _logits_case(1, dtype, 5, [1] * 5, 700, 60, 4)
    kw["mask"] = np.concatenate([kw["mask"]] * 2)
    for change in ({}, dict(mask_row=None), dict(draft=None, visible=None), dict(visible=None)):
        _check_logits(logits, None, {**kw, **change}, half)
    logits, first, kw = _logits_case(2, dtype, 2, [200, 61], 333, 40, 4, words=3)
    _check_logits(logits, first, kw, half)
    _check_logits(logits, first, {**kw, "visible": None}, half)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_in_place_strides_and_rows_of_no_sequence(dtype):
    logits, first, kw = _logits_case(3, dtype, 3, [4, 2, 3], 1003, 77, 9)
    half = dtype == "bf16"
    want = _check_logits(logits, first, kw, half)
    dev = {k: torch.from_numpy(v).to(DEV) for k, v in kw.items()}
    x = logits.to(DEV)
    assert _ops().adjust_logits(x, torch.from_numpy(first).to(DEV), out=x, **dev) is x and torch.equal(x, want)
    wide = torch.full((9, 1100), 3.0, dtype=TYPES[dtype], device=DEV)
    wide[:, 7:1010] = logits.to(DEV)
    out = torch.full((9, 1300), 3.0, dtype=TYPES[dtype], device=DEV)
    y = _ops().adjust_logits(wide[:, 7:1010], torch.from_numpy(first).to(DEV), out=out[:, 2:1005], **dev)
    assert torch.equal(y, want) and (out[:, :2] == 3).all() and (out[:, 1005:] == 3).all()
    part = _check_logits(logits, np.array([2, 4, 4, 7], np.int32), kw, half)     # rows 0, 1, 7 and 8 belong to nobody
    assert part.shape == want.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_many_sequences(dtype):
    g = np.random.default_rng(6)
    for n in (63, 64, 65, 4097):
        nodes = g.integers(0, 3, n).tolist()
        logits, first, kw = _logits_case(n, dtype, n, nodes, 37, 5, 2)
        _check_logits(logits, first, kw, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_that_are_not_finite(dtype):
    """-infinity stays, NaN stays where it is allowed, and nothing is left where the mask forbids."""
    logits, first, kw = _logits_case(4, dtype, 2, [3, 3], 300, 50, 6)
    logits[:, 10:20], logits[:, 20:30], logits[:, 30:40] = -INF, INF, NAN
    logits[0], logits[4] = NAN, -INF
    kw["mask_row"][:] = [0, 1, -1, 2, -1, 0]
    got = _check_logits(logits, first, kw, dtype == "bf16")
    assert (got[0] == -INF).any() and got[0].isnan().any()
    kw["mask"][:] = 0
    kw["mask_row"][:] = 1
    assert (_check_logits(logits, first, kw, dtype == "bf16") == -INF).all()


def test_logits_of_a_long_history_and_a_large_vocabulary():
    g = np.random.default_rng(5)
    B, V, L = 2, 128256, 100000
    logits = torch.from_numpy(g.standard_normal((B, V)).astype(np.float32))
    kw = dict(tokens=(g.random((B, L)) ** 4 * V).astype(np.int32), n_prompt=np.array([0, 50000], np.int32), repetition=np.array([1.3, 0.7], np.float32),
              frequency=np.array([0.01, -0.02], np.float32), presence=np.array([0.5, 0.0], np.float32))
    kw["tokens"][0, :70000] = 17                          # one token more often than 16 bits hold
    _check_logits(logits, None, kw, False)


# ---------------------------------------------------------------------------------------- together, streams, graphs
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rounds_of_drafted_trees(dtype):
    """Three rounds as they are used: append the trees, attend in two layers, adjust the logits, walk the trees, keep the paths.  The committed keys of a
    round are those of its accepted tokens in order, whatever pages they lie in."""
    g = torch.Generator().manual_seed(31)
    ops, dt = _ops(), TYPES[dtype]
    B, H, KVH, dh, page, layers, V = 3, 4, 2, 64, 8, 2, 211
    width = (H + 2 * KVH) * dh
    pages = 64
    keys, values = (torch.randn(layers, pages, KVH, page, dh, generator=g).to(dt).to(DEV) for _ in range(2))
    cache = ops.PagedCache(keys, values)
    table = torch.randperm(pages, generator=g)[:B * 12].reshape(B, 12).to(torch.int32).to(DEV)
    emb = torch.randn(layers, V, width, generator=g).to(DEV)            # a token's projections in every layer
    head = (torch.randn(H * dh, V, generator=g) / 8).to(DEV)
    freq = 1e4 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    committed = [torch.randint(0, V, (n,), generator=g).tolist() for n in (9, 1, 23)]
    rep = torch.full((B,), 1.2, device=DEV)
    lens = _ints([len(c) - 1 for c in committed])         # the last token is node 0 of the next tree

    def put(layer, tokens, seq, slot, pos):
        r = emb[layer, torch.tensor(tokens, device=DEV)].to(dt)
        return cache.append(layer, r[:, H * dh:(H + KVH) * dh], r[:, (H + KVH) * dh:], table, _ints(seq), _ints(slot), q=r[:, :H * dh], pos=_ints(pos), freq=freq)

    for layer in range(layers):
        put(layer, [t for c in committed for t in c[:-1]], [b for b, c in enumerate(committed) for _ in c[:-1]], [i for c in committed for i in range(len(c) - 1)],
            [i for c in committed for i in range(len(c) - 1)])

    for turn in range(3):
        parents, tokens = [], []
        for b in range(B):
            n = int(torch.randint(1, 12, (1,), generator=g))
            parents.append([-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, n)])
            tokens.append([committed[b][-1]] + torch.randint(0, V, (n - 1,), generator=g).tolist())
        nodes = [len(p) for p in parents]
        first = _ints(np.concatenate([[0], np.cumsum(nodes)]).tolist())
        depth, bits = [], []
        for p in parents:
            d, m = [], []
            for i, q in enumerate(p):
                d.append(0 if q < 0 else d[q] + 1)
                m.append((0 if q < 0 else m[q]) | 1 << i)
            depth.append(d)
            bits += [[x] for x in m]
        vis = torch.tensor(bits, dtype=torch.int64, device=DEV)
        seq = [b for b, n in enumerate(nodes) for _ in range(n)]
        l = lens.tolist()
        slot = [l[b] + i for b, n in enumerate(nodes) for i in range(n)]
        pos = [l[b] + d for b in range(B) for d in depth[b]]
        flat = [t for x in tokens for t in x]
        y = 0
        for layer in range(layers):
            q = put(layer, flat, seq, slot, pos)
            out = cache.attend(layer, q, table, lens, first, visible=vis)
            # every node alone, on its own path laid out contiguously
            t = 0
            for b in range(B):
                for i in range(nodes[b]):
                    path = [j for j in range(i + 1) if bits[t][0] >> j & 1]
                    toks = committed[b][:-1] + [tokens[b][j] for j in path]
                    r = emb[layer, torch.tensor(toks, device=DEV)].to(dt).double().cpu().numpy()
                    half = dtype == "bf16"
                    rnd = lambda x: torch.from_numpy(x).to(dt).double()  # noqa: E731
                    at = np.arange(len(toks))
                    kk = rnd(M.turned(r[:, H * dh:(H + KVH) * dh].reshape(-1, KVH, dh), at, freq.cpu().numpy(), "halves", half)[0])
                    vv = torch.from_numpy(r[:, (H + KVH) * dh:].reshape(-1, KVH, dh))
                    qq = q[t].double().cpu().reshape(H, dh)
                    for h in range(H):
                        s = kk[:, h // 2] @ qq[h] * dh ** -0.5
                        want = torch.softmax(s, 0) @ vv[:, h // 2]
                        # keys rounded from float32 angles may differ by a step of their type: 2^-8 of a score's terms at most
                        size = float((kk[:, h // 2].abs() @ qq[h].abs()).max()) * dh ** -0.5
                        tol = (2 * M.B16 if half else 200 * M.F32) * (size + 2) * float(vv[:, h // 2].abs().max())
                        assert float((out[t].double().cpu().reshape(H, dh)[h] - want).abs().max()) <= tol
                    t += 1
            y = y + out.float()
        hist = torch.zeros(B, 64, dtype=torch.int32, device=DEV)
        for b, c in enumerate(committed):
            hist[b, :len(c) - 1] = torch.tensor(c[:-1])
        logits = ops.adjust_logits(y @ head, first, tokens=hist, n_token=lens, repetition=rep, draft=_ints(flat), visible=vis)
        best = logits.argmax(dim=1).tolist()
        paths, kept, at = [], [], 0
        for b in range(B):
            i, path = 0, [0]
            while True:
                # the walk: a child whose token is the node's choice; every other one now and then, so that paths are long
                kids = [j for j in range(nodes[b]) if parents[b][j] == i]
                hit = [j for j in kids if tokens[b][j] == best[at + i]] or (kids[-1:] if torch.rand(1, generator=g) < 0.8 else [])
                if not hit:
                    break
                i = hit[0]
                path.append(i)
            committed[b] = committed[b] + [tokens[b][j] for j in path[1:]] + [best[at + i]]
            paths.append(path + [-1] * (12 - len(path)))
            kept.append(len(path))
            at += nodes[b]
        cache.keep(table, lens, first, _ints(paths), _ints(kept))
        lens = lens + _ints(kept)
        assert lens.tolist() == [len(c) - 1 for c in committed]


def _everything(b, cache, vis, seq, slot, k, v, logits, tokens, path, n_keep, freq, q_out, y, out):
    cache.append(0, k, v, b.table, seq, slot, q=b.q, freq=freq, q_out=q_out)
    cache.attend(0, q_out, b.table, b.lens, b.first, visible=vis, out=y)
    _ops().adjust_logits(logits, b.first, tokens=tokens, repetition=logits[:b.first.shape[0] - 1, 0].abs() + 1, draft=tokens[0, :b.T].contiguous(), visible=vis, out=out)
    cache.keep(b.table, b.lens, b.first, path, n_keep)


@pytest.mark.parametrize("lens", [[60, 9, 130], [3000, 40, 700]])
@pytest.mark.parametrize("how", ["stream", "graph"])
def test_on_a_stream_and_replayed_from_a_graph(lens, how):
    """All four in a row on a stream of their own and as a graph, whose inputs change between the replays: lengths, trees, pages, histories."""
    b = Batch(41, "bf16", [max(lens)] * 3, [9, 9, 9], 8, 2, 128, 16)
    g = torch.Generator().manual_seed(1)
    T, V = b.T, 600
    state = dict(vis=b.seen(), seq=_ints([0] * 9 + [1] * 9 + [2] * 9), slot=_ints([0] * 27), k=b.normal(T, 256).bfloat16(), v=b.normal(T, 256).bfloat16(), logits=b.normal(T, V),
                 tokens=torch.randint(0, V, (3, 50), generator=g).to(torch.int32).to(DEV), path=_ints([[0, 2, 5], [1, 3, 8], [0, 1, 2]]), n_keep=_ints([3, 2, 1]),
                 freq=1e4 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device=DEV) / 128), q_out=torch.empty(T, 1024, dtype=torch.bfloat16, device=DEV),
                 y=torch.empty(T, 1024, dtype=torch.bfloat16, device=DEV), out=torch.empty(T, V, device=DEV))

    def change(i):
        now = [max(0, l - 3 * i) for l in lens]
        if i == 2:
            now = now[::-1]
        b.lens.copy_(_ints(now))
        state["slot"].copy_(_ints([n + j for n in now for j in range(9)]))
        state["vis"].copy_(b.seen())
        state["k"].copy_(b.normal(T, 256))
        state["logits"].copy_(b.normal(T, V))
        b.table.copy_(b.table[:, torch.randperm(b.table.shape[1], generator=g).to(DEV)])
        state["tokens"].copy_(torch.randint(0, V, (3, 50), generator=g))

    def run():
        _everything(b, b.cache, **state)

    side = torch.cuda.Stream()
    change(0)
    if how == "graph":
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
    for i in range(5):
        change(i)
        start = b.keys.clone(), b.values.clone()
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (b.keys, b.values, state["q_out"], state["y"], state["out"])]
        b.keys.copy_(start[0])
        b.values.copy_(start[1])
        for n in ("q_out", "y", "out"):
            state[n].fill_(-1)
        if how == "graph":
            graph.replay()
        else:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                run()
            torch.cuda.current_stream().wait_stream(side)
        for t, w in zip((b.keys, b.values, state["q_out"], state["y"], state["out"]), want):
            assert torch.equal(t.view(torch.int16), w.view(torch.int16))


def test_two_graphs_and_eager_calls_at_once():
    """Two graphs whose attention splits its keys, replayed on two streams beside eager calls: workspaces are nobody else's."""
    batches = [Batch(50 + i, "bf16", [3000 - 900 * i, 1500], [4, 7], 8, 2, 128, 32) for i in range(3)]
    outs = [torch.zeros_like(b.q) for b in batches]
    want = [b.cache.attend(0, b.q, b.table, b.lens, b.first) for b in batches]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[i]):
            batches[i].cache.attend(0, batches[i].q, batches[i].table, batches[i].lens, batches[i].first, out=outs[i])
        graphs.append(graph)
    for _ in range(10):
        for o in outs:
            o.zero_()
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        b = batches[2]
        b.cache.attend(0, b.q, b.table, b.lens, b.first, out=outs[2])
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_call_gives_the_same_bits(dtype):
    b = Batch(60, dtype, [2000, 37, 512], [16, 3, 33], 8, 4, 64, 16)
    vis = b.seen()
    want = b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis)
    for _ in range(5):
        assert torch.equal(b.cache.attend(0, b.q, b.table, b.lens, b.first, visible=vis), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, longest, most", [(65, 700, 3), (128, 40, 40), (129, 40, 3), (700, 40, 3), (1300, 3000, 2)])
def test_many_sequences(dtype, n, longest, most):
    """More sequences than a wave or a workgroup has lanes, most of them short, with one node or none, a few long ones that are split."""
    g = np.random.default_rng(n)
    lens, nodes = g.integers(0, 40, n), g.integers(0, most + 1, n)
    lens[[0, n // 2, n - 1]], nodes[[0, n // 2, n - 1]] = longest, most
    b = Batch(70, dtype, lens.tolist(), nodes.tolist(), 2, 1, 64, 8)
    b.check()
    b.check(visible=b.seen())


def test_very_many_sequences():
    """Every sequence one row, as many as need four levels of the search for it; equal to sixteen batches of them."""
    n = 1 << 19
    b = Batch(73, "bf16", [3], [1], 2, 1, 64, 8)
    table = torch.randint(0, b.keys.shape[1], (n, 1), generator=b.g).to(torch.int32).to(DEV)
    lens = torch.randint(0, 8, (n,), generator=b.g).to(torch.int32).to(DEV)
    q, first = b.normal(n, 128).bfloat16(), torch.arange(n + 1, dtype=torch.int32, device=DEV)
    y = b.cache.attend(0, q, table, lens, first)
    part = n // 16
    for i in range(0, n, part):
        assert torch.equal(y[i:i + part], b.cache.attend(0, q[i:i + part], table[i:i + part], lens[i:i + part], first[:part + 1]))
    x, rep, tokens = b.normal(n, 40), b.normal(n).abs() + 0.5, torch.randint(0, 40, (n, 3), generator=b.g).to(torch.int32).to(DEV)
    assert torch.equal(_ops().adjust_logits(x, first, tokens=tokens, repetition=rep), _ops().adjust_logits(x, tokens=tokens, repetition=rep))


@pytest.mark.parametrize("first", [[0, 9, 0, 9, 0, 9], [9, 8, 7, 3, 2, 0], [-5, 3, 100, 2, -7, 9], [5, 5, 5, 5, 5, 5]])
@pytest.mark.parametrize("copies", [1, 200])
def test_rows_that_do_not_ascend_end(first, copies):
    """What `first` says then is nobody's: outputs are not said, but every call ends and writes within its rows."""
    n = 5 * copies
    b = Batch(74, "bf16", [40], [9], 4, 2, 64, 8)
    table, lens = b.table.expand(n, -1).contiguous(), torch.full((n,), 40, dtype=torch.int32, device=DEV)
    f = _ints((first[:5] * copies) + first[5:])
    out = torch.full((9 + 2, 256), 3.0, dtype=torch.bfloat16, device=DEV)
    b.cache.attend(0, b.q, table, lens, f, out=out[1:10])
    assert (out[0] == 3).all() and (out[10] == 3).all()
    x = b.normal(9, 50)
    _ops().adjust_logits(x, f, tokens=torch.zeros(n, 2, dtype=torch.int32, device=DEV), repetition=torch.ones(n, device=DEV), draft=_ints([1] * 9))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [1, 9, 20, 70])
def test_a_table_without_columns(dtype, nodes):
    """No slot is there: zeros, and nothing is written."""
    b = Batch(72, dtype, [5, 40], [nodes, nodes], 4, 2, 64, 8)
    none = b.table[:, :0]
    assert (b.cache.attend(0, b.q, none, b.lens, b.first) == 0).all()
    assert (b.cache.attend(0, b.q, none, b.lens, b.first, visible=b.seen()) == 0).all()
    keys = b.keys.clone()
    seq, k = _ints([0] * nodes + [1] * nodes), b.q[:, :128]
    b.cache.append(0, k, k, none, seq, seq)
    b.cache.keep(none, b.lens, b.first, _ints([[0, 0], [0, 0]]), _ints([2, 2]))
    assert torch.equal(keys, b.keys)


def test_empty_batches():
    b = Batch(71, "bf16", [5], [1], 2, 1, 64, 8)
    none = torch.empty(0, 128, dtype=torch.bfloat16, device=DEV)
    assert b.cache.attend(0, none, b.table, b.lens, _ints([0, 0])).shape == (0, 128)
    assert b.cache.attend(0, none, b.table[:0], _ints([]), _ints([0])).shape == (0, 128)
    keys = b.keys.clone()
    b.cache.append(0, none[:, :64], none[:, :64], b.table, _ints([]), _ints([]))
    b.cache.keep(b.table[:0], _ints([]), _ints([0]), torch.empty(0, 3, dtype=torch.int32, device=DEV), _ints([]))
    assert torch.equal(keys, b.keys) and _ops().adjust_logits(torch.empty(0, 9, device=DEV)).shape == (0, 9)
