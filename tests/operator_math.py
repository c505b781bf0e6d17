"""Routing, experts and block norms in float64 from their definitions, and how far a kernel may be from them: every rounding counted
at its half step (float16 2^-11, bfloat16 2^-8, float32 2^-24), a float32 sum of n terms at n of them on the sum of magnitudes."""
import numpy as np

H16, B16, F32 = 2.0 ** -11, 2.0 ** -8, 2.0 ** -24
TINY16 = 2.0 ** -25          # half a step of float16 below 2^-14


def route(logits, k, score="softmax", bias=None, n_group=1, top_group=1, group_score="max", renormalize=True, scale=1.0, n_shared=0):
    logits = np.asarray(logits, np.float64)
    T, E = logits.shape
    ids = np.full((T, k + n_shared), -1, np.int64)
    w = np.zeros((T, k + n_shared))
    b = np.zeros(E) if bias is None else np.asarray(bias, np.float64)
    for t in range(T):
        l = logits[t]
        ok = l > -np.inf
        p = np.zeros(E)
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                p[ok] = 1.0 / (1.0 + np.exp(-l[ok]))
        elif ok.any():
            top = l[ok].max()
            e = np.array([1.0 if v == top else np.exp(v - top) for v in l[ok]])
            p[ok] = e / e.sum()
        key = p + b
        free = [e for e in range(E) if ok[e] and key[e] > -np.inf]
        if n_group > 1:
            per = E // n_group
            rank = {}
            for g in range(n_group):
                mine = sorted((key[e] for e in free if e // per == g), reverse=True)
                if mine:
                    rank[g] = mine[0] + (mine[1] if group_score == "sum2" and len(mine) > 1 else 0.0)
            taken = sorted(rank, key=lambda g: (-rank[g], g))[:top_group]
            free = [e for e in free if e // per in taken]
        order = sorted(free, key=lambda e: (-key[e], e))[:k]
        ids[t, :len(order)] = order
        w[t, :len(order)] = p[order]
        if renormalize and w[t].sum() > 0:
            w[t] /= w[t].sum()
        w[t] *= scale
        ids[t, k:] = E + np.arange(n_shared)
        w[t, k:] = 1.0
    return ids, w


def experts(x, ids, weights, wg, wu, w2, half):
    """float64 torch tensors on one device -> (y, bound).  half: bf16 mode (float16 operands, bfloat16 result)."""
    import torch
    d, ff = x.shape[1], wg.shape[1]
    y, bound, size = (torch.zeros_like(x) for _ in range(3))
    low = TINY16 if half else 0.0
    for e in range(wg.shape[0]):
        row, place = torch.nonzero(ids == e, as_tuple=True)
        if not row.numel():
            continue
        xe, w = x[row], weights[row, place][:, None]
        g, u = xe @ wg[e].T, xe @ wu[e].T
        ones = low * (xe.abs().sum(1, keepdim=True) + wg[e].abs().sum(1) + wu[e].abs().sum(1)) + d * low * low
        dg = (d + 2) * F32 * (xe.abs() @ wg[e].abs().T) + ones
        du = (d + 2) * F32 * (xe.abs() @ wu[e].abs().T) + ones
        s = g * torch.sigmoid(g)
        hid = s * u
        dh = 1.1 * dg * (u.abs() + du) + s.abs() * du + 8 * F32 * hid.abs()       # |silu'| < 1.1
        if half:
            dh = dh * (1 + H16) + H16 * hid.abs() + TINY16
        a = w2[e].abs()
        out = hid @ w2[e].T
        do = dh @ a.T + (ff + 2) * F32 * ((hid.abs() + dh) @ a.T) + low * (hid.abs().sum(1, keepdim=True) + a.sum(1)) + 2 * H16 * low
        y.index_add_(0, row, w * out)
        size.index_add_(0, row, w.abs() * (out.abs() + hid.abs() @ a.T))
        bound.index_add_(0, row, w.abs() * do)
    # (sums over experts may run through one accumulator: its terms' magnitudes)
    bound = bound + (ids.shape[1] * (ff + 2) + 4) * F32 * size
    return y, bound * (1 + B16) + (B16 if half else F32) * y.abs() + 1e-38


def _norm(x, dx, kind, gain, offset, eps, n):
    """float64 rows with a bound on their errors -> (norm, bound); n roundings in a sum over the row."""
    mean = x.mean(1, keepdims=True) if kind == "layer" else np.zeros((x.shape[0], 1))
    dm = (n * F32 * np.abs(x).mean(1, keepdims=True) + dx.mean(1, keepdims=True)) if kind == "layer" else np.zeros_like(mean)
    c = x - mean
    dc = dx + dm + F32 * (np.abs(c) + dx + dm)
    var = (c * c).mean(1, keepdims=True)
    dvar = (2 * np.abs(c) * dc + dc * dc).mean(1, keepdims=True) + (n + 2) * F32 * var
    r = 1.0 / np.sqrt(var + eps)
    dr = r * np.minimum(0.5 * dvar / (var + eps) * (1 + dvar / (var + eps)), 1.0) + 6 * F32 * r
    v = c * r * gain + (0.0 if offset is None else offset)
    dv = (dc * r + np.abs(c) * dr + dc * dr) * np.abs(gain) + 5 * F32 * (np.abs(c * r * gain) + (0.0 if offset is None else np.abs(offset)))
    return v, dv


def block_norm(h, y, gain, offset=None, post_gain=None, post_offset=None, gate=None, scale=1.0, eps=1e-5, kind="rms", half=False):
    """float64 arrays -> (h', its bound, out, its bound)."""
    d = h.shape[1]
    n = d / 64 + 16                                       # 64 lanes or more share a row, then a tree
    u, du = y, np.zeros_like(y)
    if post_gain is not None:
        u, du = _norm(y, du, kind, post_gain, post_offset, eps, n)
    g = 1.0 if gate is None else gate
    step = scale * g * u
    hn = h + step
    dh = np.abs(scale * g) * du + 4 * F32 * np.abs(step) + F32 * (np.abs(hn) + np.abs(scale * g) * du)
    out, do = _norm(hn, dh, kind, gain, offset, eps, n)
    return hn, dh, out, do + (B16 if half else F32) * (np.abs(out) + do) + 1e-38
