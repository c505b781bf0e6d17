"""Contexts of experts in bf16 mode, with what counts as a near decision of the router taken from the rounding itself: a decision may be
the device's own only where its distance is within four deviations of what rounding makes of it, and few may be."""
import numpy as np
import pytest
import workloads as W
import test_gpu_blocks as B

# Root mean square error of a normalised row's components, whose own is about 1.  A rounding to float16 leaves 0.4 of 2^-11 in the mean
# (2.0e-4), of which each half-block has three (rows, hidden or attended values, the product's operands), one to bfloat16 0.4 of 2^-8
# (1.6e-3), of which attention has one (keys and values in the cache).  Independent, over three layers:
# sqrt(3 * 1.6e-3^2 + 18 * 2.0e-4^2) = 2.9e-3, below 2^-8 = 3.9e-3.  The test holds the device to it.
ROW_ERROR = 2.0 ** -8
NEAR = 4.0                    # deviations


class NearChoices(B.Choices):
    """Choices whose distances are counted in deviations: distance / (ROW_ERROR |gradient of the distance by the row|)."""
    routers = ()

    def __call__(self, logits, b, bias=None):
        me = len(self.made)
        ids, w = super().__call__(logits, b, bias)
        m = self.routers[me % len(self.routers)]              # (an entry passes the layers in turn)
        p = 1.0 / (1.0 + np.exp(-logits)) if b.score == "sigmoid" else np.exp(logits - logits.max()) / np.exp(logits - logits.max()).sum()
        key = p if bias is None else p + bias
        slope = (p * (1 - p))[:, None] * m if b.score == "sigmoid" else p[:, None] * (m - p @ m)       # gradients of the keys
        per = b.n_expert // b.n_group
        first = np.argsort(-key.reshape(b.n_group, per), axis=1, kind="stable") + np.arange(b.n_group)[:, None] * per
        first = first[:, :1 if b.group_score == "max" else 2]
        rank, by = key[first].sum(axis=1), slope[first].sum(axis=1)
        order = np.argsort(-rank, kind="stable")
        moves = []
        if b.top_group < b.n_group:
            i, j = order[b.top_group - 1], order[b.top_group]
            moves.append((rank[i] - rank[j], by[i] - by[j]))
        open_ = np.isin(np.arange(b.n_expert) // per, order[:b.top_group])
        taken = np.argsort(-np.where(open_, key, -np.inf), kind="stable")
        if open_.sum() > b.top_k:
            i, j = taken[b.top_k - 1], taken[b.top_k]
            moves.append((key[i] - key[j], slope[i] - slope[j]))
        self.made[me] = min(d / (ROW_ERROR * np.linalg.norm(v)) for d, v in moves)
        return ids, w


def _routers(weights, cfg):
    return [np.asarray(weights[f"l{i}.router"], np.float64) for i in range(cfg.target.n_layer)]


@pytest.mark.parametrize("kind", ["experts", "groups"])
def test_few_decisions_are_near(kind, monkeypatch):
    """The oracle alone: the band is well below the distance of most decisions, so that it explains few wrong ones."""
    from oracle import model as om, sprinter as osp
    cfg = W.mini_config(kind, W.DT_BF16, batch=3, n_gen=12)
    dw, tw, vw = W.make_weights(cfg)
    monkeypatch.setattr(NearChoices, "routers", _routers(tw, cfg))
    c = NearChoices()
    monkeypatch.setattr(om, "take_experts", c)
    prompts, plen = W.make_prompts(cfg)
    osp.generate(om.Decoder(cfg.draft, dw), om.Decoder(cfg.target, tw), om.Verifier(vw), prompts, plen, 12, cfg.tau, cfg.temperature, cfg.seed,
                 ctx_mode=cfg.target_ctx_mode, reject_mode=cfg.reject_mode)
    far = np.asarray(c.made)
    print(kind, len(far), "decisions, distances in deviations", np.quantile(far, [0.01, 0.05, 0.1, 0.25, 0.5]).round(2), "within 4:", (far <= 4).mean())
    assert len(far) % cfg.target.n_layer == 0
    assert np.median(far) > 4 * NEAR and (far <= NEAR).mean() < 0.125


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["experts", "groups"])
@pytest.mark.parametrize("batch", [19, 3])
def test_steps_with_near_decisions_only(kind, batch, monkeypatch):
    from parity_util import Pair, close_enough, eps_of
    cfg = W.mini_config(kind, W.DT_BF16, batch=batch, n_gen=12)
    p = Pair(cfg, ver_scale=8.0)
    monkeypatch.setattr(NearChoices, "routers", _routers(p.weights[1], cfg))
    monkeypatch.setattr(B, "Choices", NearChoices)
    monkeypatch.setattr(B, "_band", lambda p: NEAR)
    outs, st = p.gpu_steps(12, debug=True)
    g = {k: np.stack([o[k2] for o in outs], axis=1) for k, k2 in
         (("tok", "committed_tok"), ("accept", "accept"), ("score", "score"), ("draft_tok", "draft_tok"))}
    rec, recs, moved = B._replay(p, g, 12, outs, monkeypatch)
    eps, off, size, n = eps_of(cfg), 0.0, 0.0, 0
    for s, o in enumerate(outs):
        for i, b in enumerate(np.flatnonzero(o["accept"] == 0)):
            want = recs[b]["target_hidden"][s][0]
            assert close_enough(o["target_hidden"][i], want, eps).all() and close_enough(o["target_logits"][i], recs[b]["target_logits"][s][0], eps).all()
            off, size, n = off + ((o["target_hidden"][i] - want) ** 2).sum(), size + (np.asarray(want, np.float64) ** 2).sum(), n + want.size
    made = cfg.target.n_layer * sum(int(p.plen[b]) - 1 + int((g["accept"][b] == 0).sum()) for b in range(batch))
    print(kind, batch, "row error", np.sqrt(off / size), "of", np.sqrt(size / n), "decisions", made, "moved", moved, flush=True)
    assert np.sqrt(off / size) <= ROW_ERROR
    assert moved <= max(1, 0.02 * made)                   # (4 - 8 % are near; of those within d deviations fewer than half go the other way)
    p.close()
