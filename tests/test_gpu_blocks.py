"""Contexts whose models have described blocks (experts, norms behind attention and feed-forward, gates, residual scale), against the
oracle replayed on their history, through every forward pass there is: prefill, decode steps, full-prefix work lists, speculative rounds."""
from dataclasses import replace
import numpy as np
import pytest
import workloads as W

pytestmark = pytest.mark.gpu


def _pair(cfg, **kw):
    from parity_util import Pair
    return Pair(cfg, **kw)


class Choices:
    """Stands in for the oracle's take_experts: notes every decision with the nearest other one, and takes that one where told to.

    bf16 mode rounds what the router reads, so where two keys (or two groups' ranks) lie closer than that moves them the device may take
    the other one, and everything behind it differs by more than a rounding.  Such a decision is shown, not assumed: the definition with
    that one decision changed has to give the device's logits and hidden states within the usual tolerance."""

    def __init__(self, other=()):
        from oracle import model as om
        self.take, self.other, self.made = om.take_experts, dict.fromkeys(other), []

    def __call__(self, logits, b, bias=None):
        ids, w = self.take(logits, b, bias)
        p = 1.0 / (1.0 + np.exp(-logits)) if b.score == "sigmoid" else np.exp(logits - logits.max()) / np.exp(logits - logits.max()).sum()
        key = p if bias is None else p + bias
        per = b.n_expert // b.n_group
        best = -np.sort(-key.reshape(b.n_group, per), axis=1)
        rank = best[:, 0] if b.group_score == "max" else best[:, :2].sum(axis=1)
        order = np.argsort(-rank, kind="stable")
        moves = []                                            # (distance, the groups then open, the expert then left out)
        if b.top_group < b.n_group:
            moves.append((rank[order[b.top_group - 1]] - rank[order[b.top_group]], np.append(order[:b.top_group - 1], order[b.top_group]), None))
        open_ = np.isin(np.arange(b.n_expert) // per, order[:b.top_group])
        rest = [e for e in np.flatnonzero(open_) if e not in ids]
        if rest:
            moves.append((key[ids[-1]] - key[rest].max(), order[:b.top_group], ids[-1]))
        me = len(self.made)
        far, groups, left_out = min(moves, key=lambda m: m[0])
        self.made.append(far)
        if me in self.other:
            k2 = np.where(np.isin(np.arange(b.n_expert) // per, groups), key, -np.inf)
            if left_out is not None:
                k2[left_out] = -np.inf
            ids = np.argsort(-k2, kind="stable")[:b.top_k]
            w = p[ids] / (p[ids].sum() if b.renormalize else 1.0) * b.route_scale
        return ids, w


def _band(p):
    """How far rounding may move a key: |d logit| <= |w|_2 |d x|_2 (Cauchy-Schwarz) with every component of x within the tolerance of
    hidden states, and a score moves by at most a quarter of its logit; two keys move towards each other."""
    from parity_util import eps_of
    rows = [np.linalg.norm(v, axis=1).max() for k, v in p.weights[1].items() if k.endswith(".router")]
    return 2 * max(rows) * eps_of(p.cfg) * np.sqrt(p.cfg.target.d_model) / 4


def _replay(p, g, n, outs, monkeypatch):
    """The oracle on the GPU's history, row by row, with the decisions that lie within the band as the GPU has taken them."""
    from oracle import model as om
    from parity_util import close_enough, eps_of
    eps, recs, moved = eps_of(p.cfg), [], 0

    def first_apart(rec, b):
        for s, o in enumerate(outs):
            rej = list(np.flatnonzero(o["accept"] == 0))
            if b in rej and not (close_enough(o["target_logits"][rej.index(b)], rec["target_logits"][s][0], eps).all() and
                                 close_enough(o["target_hidden"][rej.index(b)], rec["target_hidden"][s][0], eps).all()):
                return s
        return n

    def run(b, other):
        c = Choices(other)
        with monkeypatch.context() as m:
            m.setattr(om, "take_experts", c)
            return p.oracle(n, forced=dict(tok=g["tok"], accept=g["accept"]), rows=[b], keep_logits=True), c

    for b in range(len(p.plen)):
        other = ()
        rec, c = run(b, other)
        while (s := first_apart(rec, b)) < n:
            entries = p.plen[b] - 1 + int((g["accept"][b, :s + 1] == 0).sum())        # what the target has read by then
            near = sorted((far, i) for i, far in enumerate(c.made[:entries * p.cfg.target.n_layer]) if far <= _band(p) and i not in other)
            for far, i in near[:12]:
                r2, c2 = run(b, other + (i,))
                if first_apart(r2, b) > s:
                    rec, c, other = r2, c2, other + (i,)
                    print("row", b, "step", s, "took the other expert, keys apart by", far, flush=True)
                    break
            else:
                raise AssertionError(f"row {b} differs from step {s} on, and no near decision explains it")
        moved += len(other)
        recs.append(rec)
    whole = {k: np.concatenate([r[k] for r in recs]) for k in recs[0] if isinstance(recs[0][k], np.ndarray) and recs[0][k].ndim == 2 and
             recs[0][k].shape[0] == 1}
    return whole, recs, moved


@pytest.mark.parametrize("kind", ["experts", "groups"])
@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
@pytest.mark.parametrize("batch", [19, 3])
def test_steps(kind, dtype, batch, monkeypatch):
    from parity_util import compare_replay, close_enough, eps_of
    cfg = W.mini_config(kind, dtype, batch=batch, n_gen=12)
    p = _pair(cfg, ver_scale=8.0)
    outs, st = p.gpu_steps(12, debug=True)
    g = {k: np.stack([o[k2] for o in outs], axis=1) for k, k2 in
         (("tok", "committed_tok"), ("accept", "accept"), ("score", "score"), ("draft_tok", "draft_tok"))}
    rec, recs, moved = _replay(p, g, 12, outs, monkeypatch)
    print(kind, dtype, compare_replay(cfg, g, rec), "decisions moved", moved, flush=True)
    eps = eps_of(cfg)
    worst = 0.0
    for s, o in enumerate(outs):
        rej = list(np.flatnonzero(o["accept"] == 0))
        for b in range(batch):
            assert close_enough(o["draft_logits"][b], recs[b]["draft_logits"][s][0], eps).all()
            assert close_enough(o["draft_hidden"][b], recs[b]["draft_hidden"][s][0], eps).all()
        for i, b in enumerate(rej):
            worst = max(worst, np.abs(o["target_hidden"][i] - recs[b]["target_hidden"][s][0]).max())
            assert close_enough(o["target_logits"][i], recs[b]["target_logits"][s][0], eps).all()
            assert close_enough(o["target_hidden"][i], recs[b]["target_hidden"][s][0], eps).all()
    print("max |target hidden diff|", worst, flush=True)
    assert moved == 0 or dtype == W.DT_BF16
    assert 0 < st["sum_rejected"] < 12 * batch
    g2, _ = p.gpu_generate(12)                           # the same again, bit for bit
    for k in ("tok", "accept", "draft_tok"):
        assert np.array_equal(g2[k], g[k]), k
    p.close()


@pytest.mark.parametrize("kind", ["experts", "groups"])
@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
def test_full_prefix(kind, dtype):
    from parity_util import compare_replay
    cfg = replace(W.mini_config(kind, dtype, n_gen=10), target_ctx_mode=W.CTX_FULL_PREFIX, chunk_rows=64)
    p = _pair(cfg, ver_scale=8.0)
    g, _ = p.gpu_generate(10)
    rec = p.oracle(10, forced=dict(tok=g["tok"], accept=g["accept"]))
    print(compare_replay(cfg, g, rec), flush=True)
    p.close()


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
def test_speculative_rounds(dtype):
    from oracle import sd_baseline as osd
    from parity_util import compare_sd_rounds, sd_rounds_to_lists
    cfg = replace(W.mini_config("experts", dtype, batch=5), sd_gamma=3)
    p = _pair(cfg)
    p.gpu.prefill(p.prompts, p.plen)
    g = {k: v.cpu().numpy() for k, v in p.gpu.sd_generate(3, 4).items()}
    lists, n_acc, draft = sd_rounds_to_lists(g)
    rec = osd.sd_generate(p.draft, p.target, p.prompts, p.plen, 4, 3, cfg.temperature, cfg.seed, rows=list(range(cfg.batch)),
                          forced=dict(tok=lists, n_acc=n_acc, draft=draft))
    print(compare_sd_rounds(cfg, g, rec), flush=True)
    p.close()


@pytest.mark.parametrize("layers", [1, 2])
def test_a_draft_of_experts_and_few_layers(layers):
    from parity_util import compare_replay
    cfg = W.mini_config("groups", W.DT_F32, batch=7, n_gen=8)
    cfg = replace(cfg, draft=replace(cfg.draft, n_layer=layers, blocks=W.BlockCfg(4, 1, 72, "sigmoid", n_shared=2, gate=True, residual_scale=0.7)),
                  target=replace(cfg.target, n_layer=layers))
    p = _pair(cfg, ver_scale=8.0)
    g, _ = p.gpu_generate(8)
    print(compare_replay(cfg, g, p.oracle(8, forced=dict(tok=g["tok"], accept=g["accept"]))), flush=True)
    p.close()


def test_a_block_without_anything_is_the_dense_one():
    """A BlockCfg that describes nothing runs through other launches than a model without one, and agrees with the same oracle."""
    from parity_util import compare_replay
    base = W.mini_config("llama", W.DT_BF16, n_gen=8)
    cfg = replace(base, draft=replace(base.draft, blocks=W.BlockCfg()), target=replace(base.target, blocks=W.BlockCfg()))
    p = _pair(cfg, ver_scale=8.0)
    g, _ = p.gpu_generate(8)
    print(compare_replay(cfg, g, p.oracle(8, forced=dict(tok=g["tok"], accept=g["accept"]))), flush=True)
    p.close()


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
def test_the_experts_matter(dtype):
    """Weights of experts in another order give other logits: the parity above would see a wrong expert."""
    cfg = W.mini_config("experts", dtype, batch=4, n_gen=2)
    dw, tw, vw = W.make_weights(cfg)
    p = _pair(cfg, weights=(dw, tw, vw))
    p.gpu.set_tau(1.5)
    a = p.gpu_steps(1)[0][0]
    p.close()
    other = {k: (np.roll(v, 1, axis=0) if v.ndim == 3 else v) for k, v in tw.items()}
    p = _pair(cfg, weights=(dw, other, vw))
    p.gpu.set_tau(1.5)
    b = p.gpu_steps(1)[0][0]
    p.close()
    from parity_util import eps_of
    assert np.abs(a["target_hidden"] - b["target_hidden"]).max() > 4 * eps_of(cfg)
