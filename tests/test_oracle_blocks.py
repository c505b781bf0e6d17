"""The oracle's described blocks: experts, norms behind attention and feed-forward, gates, residual scale."""
from dataclasses import replace
import numpy as np
import pytest
import workloads as W
from oracle import model as om
import operator_math as M


@pytest.mark.parametrize("kind", ["experts", "groups"])
def test_cached_steps_equal_whole_sequences(kind):
    cfg = W.mini_config(kind, W.DT_F32)
    for m, w in zip((cfg.draft, cfg.target), W.make_weights(cfg)):
        d = om.Decoder(m, w)
        tokens = np.arange(7) * 13 % m.vocab
        hf, logits = d.forward_full(tokens)
        caches = [d.new_cache()]
        for t, tok in enumerate(tokens):
            h, l = d.step([tok], [t], caches)
            assert np.allclose(h[0], hf[t], rtol=1e-10, atol=1e-12) and np.allclose(l[0], logits[t], rtol=1e-10, atol=1e-12)


def _dense(**kw):
    m = replace(W.mini_config("llama", W.DT_F32).target, **kw)
    return m, W.make_model_weights(m, 5, False)


def test_equal_experts_are_the_dense_block():
    m, w = _dense()
    b = W.BlockCfg(4, 2, m.d_ff, score="sigmoid")
    mw = dict(w)
    for i in range(m.n_layer):
        for n in ("wg", "wu", "w2"):
            mw[f"l{i}.{n}"] = np.stack([w[f"l{i}.{n}"]] * 4)
        mw[f"l{i}.router"] = np.random.default_rng(i).standard_normal((4, m.d_model)).astype(np.float32)
    tokens = np.array([3, 900, 17, 4])
    a = om.Decoder(m, w).forward_full(tokens)[1]
    assert np.allclose(om.Decoder(replace(m, blocks=b), mw).forward_full(tokens)[1], a, rtol=1e-9, atol=1e-11)
    # the hidden columns dealt out to shared experts add up to the dense block (routed ones of weight zero beside them)
    half = m.d_ff // 2
    sw = dict(mw)
    for i in range(m.n_layer):
        g, u, d = (w[f"l{i}.{n}"] for n in ("wg", "wu", "w2"))
        sw[f"l{i}.router"] = mw[f"l{i}.router"][:1]
        sw[f"l{i}.wg"], sw[f"l{i}.wu"] = (np.stack([x[:half] * 0, x[:half], x[half:]]) for x in (g, u))
        sw[f"l{i}.w2"] = np.stack([d[:, :half], d[:, :half], d[:, half:]])
    s = replace(m, blocks=W.BlockCfg(1, 1, half, n_shared=2))
    assert np.allclose(om.Decoder(s, sw).forward_full(tokens)[1], a, rtol=1e-9, atol=1e-11)


def test_gates_norms_and_scale():
    m, w = _dense()
    tokens = np.array([3, 900, 17, 4])
    gw = dict(w)
    for i in range(m.n_layer):
        gw[f"l{i}.gate1"] = gw[f"l{i}.gate2"] = np.full(m.d_model, 2.0, np.float32)
    a = om.Decoder(m, w).forward_full(tokens)[1]
    twice = om.Decoder(replace(m, blocks=W.BlockCfg(gate=True, residual_scale=0.5)), gw).forward_full(tokens)[1]
    assert np.allclose(twice, a, rtol=1e-10, atol=1e-12)
    # a post norm makes what a block returns independent of its scale
    pw = {k: (v * 8 if k.endswith((".wo", ".w2")) else v) for k, v in w.items()}
    for x in (w, pw):
        for i in range(m.n_layer):
            x[f"l{i}.post1.g"] = x[f"l{i}.post2.g"] = np.ones(m.d_model, np.float32)
    pm = replace(m, blocks=W.BlockCfg(post_norm=True), norm_eps=0.0)
    assert np.allclose(om.Decoder(pm, w).forward_full(tokens)[1], om.Decoder(pm, pw).forward_full(tokens)[1], rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("kind", ["experts", "groups"])
def test_routing_is_the_operators_definition(kind):
    b = W.mini_config(kind).target.blocks
    g = np.random.default_rng(3)
    logits, bias = g.standard_normal((50, b.n_expert)), g.standard_normal(b.n_expert) * 0.1
    for bi in (None, bias):
        ids, w = M.route(logits, b.top_k, score=b.score, bias=bi, n_group=b.n_group, top_group=b.top_group, group_score=b.group_score,
                         renormalize=b.renormalize, scale=b.route_scale)
        for r in range(50):
            oi, ow = om.take_experts(logits[r], b, bi)
            assert np.array_equal(oi, ids[r]) and np.allclose(ow, w[r], rtol=1e-13)
