"""The operators whose time is tracked: routing to experts, the experts' products, and the norms around a block.

`run` is one call of one operator.  In its plain form it is elementary torch in float32 (routing scores in float64: whether an expert
is taken is decided next to a border); with `own` set it is the framework's entry point.

    route    T rows of E logits -> the ids and weights of each row's top_k experts
    experts  y[t] = sum_j w[t, j] W2[e] (silu(Wg[e] x[t]) * (Wu[e] x[t])), e = ids[t, j]
    norm     u = norm(y) or y;  h' = h + scale * gate * u;  out = norm(h')

Widths are those of the workloads' models (256 / 512 / 768 / 1600 / 2048 / 4096 columns, hidden widths 704 - 14336) and eighths of
them for many small experts; the numbers of experts are generic.
"""
import math

import torch

own = False

DEV = "cuda"


# --------------------------------------------------------------------------------------------------------------- cases
def _route(name, rows, experts, top_k, score="softmax", bias=False, groups=1, top_groups=1, group_score="max", renorm=True, scale=1.0,
           shared=0, masked=0.0):
    return dict(name=name, op="route", rows=rows, experts=experts, top_k=top_k, score=score, bias=bias, groups=groups,
                top_groups=top_groups, group_score=group_score, renorm=renorm, scale=scale, shared=shared, masked=masked)


def _experts(name, dtype, rows, experts, top_k, d, ff, dropped=0.0, skew=0.5):
    return dict(name=name, op="experts", dtype=dtype, rows=rows, experts=experts, top_k=top_k, d=d, ff=ff, dropped=dropped, skew=skew)


def _norm(name, dtype, rows, d, kind="rms", post=True, gate="none", scale=1.0):
    return dict(name=name, op="norm", dtype=dtype, rows=rows, d=d, kind=kind, post=post, gate=gate, scale=scale)


def listed():
    return [
        # one token of one request: latency alone
        _route("route_token", 1, 8, 2),
        # a decode batch over many small experts, the score of the weights not renormalised
        _route("route_batch", 64, 64, 6, renorm=False, shared=2),
        # a prompt chunk with sigmoid scores, a balance bias and groups
        _route("route_groups", 4096, 256, 8, score="sigmoid", bias=True, groups=8, top_groups=4, group_score="sum2", scale=2.5),
        # the largest chunk, a ragged end, one expert in ten masked off per row
        _route("route_prompt", 16381, 64, 8, masked=0.1),
        # the float32 mode: a ragged batch of the smallest pair's target
        _experts("experts_f32_batch24", "f32", 24, 8, 2, 512, 2048),
        # one interactive request to a wide model: two experts' weights, once
        _experts("experts_token", "bf16", 1, 8, 2, 4096, 14336),
        # a decode batch over many small experts
        _experts("experts_batch16", "bf16", 16, 64, 8, 2048, 1024),
        # the rows a decode batch rejects, a few of them without any expert on this device
        _experts("experts_ragged61", "bf16", 61, 8, 2, 4096, 14336, dropped=0.05),
        # a prompt chunk over many small experts, unevenly used
        _experts("experts_many1789", "bf16", 1789, 64, 8, 2048, 1024, skew=1.0),
        # a full prompt chunk of the wide model
        _experts("experts_prompt", "bf16", 4096, 8, 2, 4096, 14336),
        # one token's residual row
        _norm("norm_token", "bf16", 1, 4096),
        # a full prompt chunk with a gain per column
        _norm("norm_prompt", "bf16", 4096, 4096, gate="column", scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route", "route", "experts", "experts", "experts", "norm"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        per = _log_int(rng, 2, 256 // groups)
        top_groups = rng.randint(1, groups)
        c = _route("", _log_int(rng, 1, 16384), groups * per, rng.randint(1, min(8, top_groups * per)),
                   score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups,
                   group_score=rng.choice(("max", "sum2")), renorm=rng.random() < 0.7, scale=rng.choice((1.0, 2.5)),
                   shared=rng.choice((0, 0, 1, 2)), masked=rng.choice((0.0, 0.0, 0.1)))
        while c["rows"] * c["experts"] > 16384 * 64:      # no more than the largest listed one
            c["rows"] = (c["rows"] + 1) // 2
    elif op == "experts":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        experts = _log_int(rng, 4, 64)
        d = 8 * _log_int(rng, 32, 512)
        ff = 8 * _log_int(rng, 16, 1792)
        while experts * d * ff > (8 * 4096 * 14336 if dtype == "bf16" else 8 * 1024 * 4096):
            if ff > 128:
                ff = max(128, ff // 16 * 8)
            else:
                d = max(256, d // 16 * 8)
        top_k = rng.randint(1, min(8, experts))
        rows = _log_int(rng, 1, 4096 if dtype == "bf16" else 512)
        while rows * top_k > 8192:
            rows = (rows + 1) // 2
        c = _experts("", dtype, rows, experts, top_k, d, ff, dropped=rng.choice((0.0, 0.05)), skew=rng.choice((0.2, 0.5, 1.0)))
    else:
        c = _norm("", rng.choice(("bf16", "bf16", "f32")), _log_int(rng, 1, 4096), rng.choice((1, 8)) * _log_int(rng, 32, 512),
                  kind=rng.choice(("rms", "rms", "layer")), post=rng.random() < 0.7, gate=rng.choice(("none", "column", "row", "both")),
                  scale=rng.choice((1.0, 0.5, 0.22)))
    del c["name"]
    return c


# -------------------------------------------------------------------------------------------------------------- inputs
def _make(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.empty(shape, dtype=dtype, device=DEV)
        return t.normal_(mean, std, generator=g)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    s = dict(case=case)
    T = case["rows"]
    if case["op"] == "route":
        E = case["experts"]
        # a trained router: some experts are liked more than others, and rows differ in how sure they are
        s["logits"] = normal(T, E) * (0.5 + 2.0 * uniform(T, 1)) + normal(E, std=0.5)
        if case["masked"] > 0:
            s["logits"] = torch.where(uniform(T, E) < case["masked"], torch.full((), -math.inf, device=DEV), s["logits"])
        s["bias"] = normal(E, std=0.05) if case["bias"] else None
        return s
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    d = case["d"]
    if case["op"] == "experts":
        E, ff, k = case["experts"], case["ff"], case["top_k"]
        # weights are bfloat16 values in both modes' ranges: N(0, 1/sqrt(fan in)) keeps every product of order one
        s["wg"] = normal(E, ff, d, std=d ** -0.5, dtype=dt)
        s["wu"] = normal(E, ff, d, std=d ** -0.5, dtype=dt)
        s["w2"] = normal(E, d, ff, std=ff ** -0.5, dtype=dt)
        s["x"] = normal(T, d, dtype=dt)                                  # a normalised row
        logits = normal(T, E) + normal(E, std=case["skew"])
        top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
        s["weights"] = torch.softmax(top[:, :k], dim=1).contiguous()
        ids = ids[:, :k].to(torch.int32)
        if case["dropped"] > 0:                                          # experts of another device
            ids = torch.where(uniform(T, k) < case["dropped"], torch.full((), -1, dtype=torch.int32, device=DEV), ids)
        s["ids"] = ids.contiguous()
        return s
    # the residual stream grows along the depth and has a few large columns
    s["h"] = normal(T, d, std=3.0) * (1.0 + 8.0 * (uniform(d) < 0.01))
    s["y"] = normal(T, d, std=0.7, dtype=dt)
    layer = case["kind"] == "layer"
    s["post_gain"] = normal(d, std=0.02, mean=1.0) if case["post"] else None
    s["post_offset"] = normal(d, std=0.02) if case["post"] and layer else None
    s["gain"] = normal(d, std=0.02, mean=1.0)
    s["offset"] = normal(d, std=0.02) if layer else None
    s["gate"] = {"none": None, "column": normal(d, std=0.3), "row": uniform(T, 1), "both": normal(T, d, std=0.3)}[case["gate"]]
    return s


def prepare(case, seed):
    s = _make(case, seed)
    if own and case["op"] == "experts":
        from paper_2502_04557_amd import operators
        s["handle"] = operators.Experts(s["wg"], s["wu"], s["w2"])       # laid out once, as at load time
    return s


# ------------------------------------------------------------------------------------------------------- one pass
EPS = 1e-5


def _plain_route(s):
    c = s["case"]
    logits = s["logits"].double()
    T, E = logits.shape
    there = logits > -math.inf
    zero = logits.new_zeros(())
    low = logits.new_full((), -math.inf)
    if c["score"] == "softmax":
        top = torch.where(there, logits, low).amax(dim=1, keepdim=True)
        e = torch.where(there, torch.exp(logits - top), zero)
        p = torch.where(there, e / e.sum(dim=1, keepdim=True), zero)
    else:
        p = torch.where(there, 1.0 / (1.0 + torch.exp(-logits)), zero)
    key = p if s["bias"] is None else p + s["bias"].double()
    key = torch.where(there, key, low)
    if c["groups"] > 1:
        g = key.view(T, c["groups"], E // c["groups"])
        best = torch.sort(g, dim=2, descending=True)[0]
        rank = best[:, :, 0]
        if c["group_score"] == "sum2" and g.shape[2] > 1:
            rank = rank + torch.where(best[:, :, 1] > low, best[:, :, 1], zero)
        taken = torch.sort(rank, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        keep = torch.zeros_like(rank).scatter_(1, taken, 1.0) > 0
        key = torch.where(keep[:, :, None], g, low).reshape(T, E)
    best, order = torch.sort(key, dim=1, descending=True, stable=True)
    best, order = best[:, :c["top_k"]], order[:, :c["top_k"]]
    some = best > low
    w = torch.where(some, p.gather(1, order), zero)
    if c["renorm"]:
        total = w.sum(dim=1, keepdim=True)
        w = torch.where(total > 0, w / total, zero)
    w = w * c["scale"]
    ids = torch.where(some, order, -1)
    if c["shared"]:
        more = torch.arange(E, E + c["shared"], device=ids.device).expand(T, c["shared"])
        ids = torch.cat([ids, more], dim=1)
        w = torch.cat([w, torch.ones_like(more, dtype=w.dtype)], dim=1)
    return ids.to(torch.int32), w.float()


def _plain_experts(s):
    x, ids, weights = s["x"], s["ids"], s["weights"]
    xf = x.float()
    y = torch.zeros_like(xf)
    for e in range(s["case"]["experts"]):
        row, place = torch.nonzero(ids == e, as_tuple=True)
        if row.numel() == 0:
            continue
        xe = xf[row]
        gate = xe @ s["wg"][e].float().t()
        up = xe @ s["wu"][e].float().t()
        hid = gate / (1.0 + torch.exp(-gate)) * up
        y.index_add_(0, row, (hid @ s["w2"][e].float().t()) * weights[row, place][:, None])
    return y.to(x.dtype)


def _plain_norm_of(x, kind, gain, offset):
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * gain
    x = x - x.mean(dim=1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * gain + offset


def _plain_norm(s):
    c = s["case"]
    u = s["y"].float()
    if c["post"]:
        u = _plain_norm_of(u, c["kind"], s["post_gain"], s["post_offset"])
    if s["gate"] is not None:
        u = u * s["gate"]
    h = s["h"] + c["scale"] * u
    return h, _plain_norm_of(h, c["kind"], s["gain"], s["offset"]).to(s["y"].dtype)


def run(state):
    c = state["case"]
    if not own:
        return {"route": _plain_route, "experts": _plain_experts, "norm": _plain_norm}[c["op"]](state)
    from paper_2502_04557_amd import operators
    if c["op"] == "route":
        return operators.route(state["logits"], c["top_k"], score=c["score"], bias=state["bias"], n_group=c["groups"],
                               top_group=c["top_groups"], group_score=c["group_score"], renormalize=c["renorm"], scale=c["scale"],
                               n_shared=c["shared"])
    if c["op"] == "experts":
        return state["handle"](state["x"], state["ids"], state["weights"])
    return operators.block_norm(state["h"], state["y"], state["gain"], offset=state["offset"], post_gain=state["post_gain"],
                                post_offset=state["post_offset"], gate=state["gate"], scale=c["scale"], eps=EPS, kind=c["kind"])


# ------------------------------------------------------------------------------------------------------------- measures
def work(case):
    T = case["rows"]
    if case["op"] == "route":
        E, n = case["experts"], case["top_k"] + case["shared"]
        return {"bytes": 4 * T * E + 4 * E * case["bias"] + 8 * T * n, "flops": 10 * T * E}
    size = 2 if case["dtype"] == "bf16" else 4
    d = case["d"]
    if case["op"] == "experts":
        E, k, ff = case["experts"], case["top_k"], case["ff"]
        pairs = T * k * (1.0 - case["dropped"])
        used = E * (1.0 - (1.0 - k / E) ** T)            # experts that some row names, were all liked alike
        return {"bytes": int(3 * used * d * ff * size + 2 * T * d * size + 8 * T * k), "flops": int(6 * pairs * d * ff)}
    gate = {"none": 0, "column": d, "row": T, "both": T * d}[case["gate"]]
    gains = d * (1 + case["post"]) * (2 if case["kind"] == "layer" else 1)
    return {"bytes": T * d * (8 + 2 * size) + 4 * (gate + gains), "flops": T * d * (12 if case["post"] else 7)}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_route(s):
    c = s["case"]
    T, E, k = c["rows"], c["experts"], c["top_k"]
    logit = s["logits"].to(torch.float64).cpu()
    off = ~(logit > -math.inf)
    if c["score"] == "softmax":
        p = torch.exp(logit.masked_fill(off, -math.inf) - torch.logsumexp(logit.masked_fill(off, -math.inf), dim=1, keepdim=True))
    else:
        p = torch.exp(-torch.log1p(torch.exp(-logit)))
    p = p.masked_fill(off, 0.0)
    key = (p + (0.0 if s["bias"] is None else s["bias"].to(torch.float64).cpu())).masked_fill(off, -math.inf)
    if c["groups"] > 1:
        per = E // c["groups"]
        rank = torch.stack([key[:, i * per:(i + 1) * per].amax(dim=1) for i in range(c["groups"])], dim=1)
        if c["group_score"] == "sum2":
            for i in range(c["groups"]):
                part = key[:, i * per:(i + 1) * per].clone()
                part.scatter_(1, part.argmax(dim=1, keepdim=True), -math.inf)
                second = part.amax(dim=1)
                rank[:, i] += torch.where(second.isinf(), torch.zeros_like(second), second)
        alive = torch.zeros(T, c["groups"], dtype=torch.bool)
        for _ in range(c["top_groups"]):
            best = rank.masked_fill(alive, -math.inf)
            pick = torch.where(alive, -1, torch.arange(c["groups"], 0, -1)[None, :])      # lowest index among the largest
            pick = torch.where(best == best.amax(dim=1, keepdim=True), pick, -1).argmax(dim=1, keepdim=True)
            alive.scatter_(1, pick, True)
        key = key.masked_fill(~alive.repeat_interleave(per, dim=1), -math.inf)
    ids = torch.full((T, k), -1, dtype=torch.int64)
    w = torch.zeros(T, k, dtype=torch.float64)
    left = key.clone()
    place = torch.arange(E, 0, -1)[None, :]
    for j in range(k):
        top = left.amax(dim=1, keepdim=True)
        pick = torch.where(left == top, place, 0).argmax(dim=1, keepdim=True)
        some = ~torch.isinf(top)
        ids[:, j:j + 1] = torch.where(some, pick, -1)
        w[:, j:j + 1] = torch.where(some, p.gather(1, pick), torch.zeros_like(top))
        left.scatter_(1, pick, -math.inf)
    if c["renorm"]:
        w = w / w.sum(dim=1, keepdim=True).clamp_min(1e-300)
    w = w * c["scale"]
    for j in range(c["shared"]):
        ids = torch.cat([ids, torch.full((T, 1), E + j)], dim=1)
        w = torch.cat([w, torch.ones(T, 1, dtype=torch.float64)], dim=1)
    return ids, w


def _exact_experts(s):
    c = s["case"]
    x = s["x"].to(torch.float64)
    share = torch.zeros(c["rows"], c["experts"] + 1, dtype=torch.float64, device=x.device)
    share.scatter_add_(1, s["ids"].long() % (c["experts"] + 1), s["weights"].double())     # -1: the last column
    y = torch.zeros_like(x)
    for e in range(c["experts"]):
        rows = share[:, e].nonzero()[:, 0]
        if rows.numel():
            a = torch.matmul(x[rows], s["wg"][e].double().T)
            a = a * torch.sigmoid(a) * torch.matmul(x[rows], s["wu"][e].double().T)
            y[rows] += share[rows, e, None] * torch.matmul(a, s["w2"][e].double().T)
    return y


def _exact_norm(s):
    c = s["case"]

    def normed(v, gain, offset):
        if c["kind"] == "layer":
            var, mean = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
            return (v - mean) / torch.sqrt(var + EPS) * gain.double() + offset.double()
        return v / torch.sqrt(v.pow(2).sum(dim=1, keepdim=True) / v.shape[1] + EPS) * gain.double()

    u = s["y"].double()
    if s["post_gain"] is not None:
        u = normed(u, s["post_gain"], s["post_offset"])
    h = s["h"].double() + (u if s["gate"] is None else s["gate"].double() * u) * c["scale"]
    return h, normed(h, s["gain"], s["offset"])


def exact(case, seed):
    return {"route": _exact_route, "experts": _exact_experts, "norm": _exact_norm}[case["op"]](_make(case, seed))
