"""A round of drafted trees over a cache in pages in float64 from the operators' definitions, and how far a kernel may be from them: every
rounding counted at its half step (bfloat16 2^-8, float32 2^-24), a float32 sum of n terms at n of them on the sum of magnitudes."""
import numpy as np
import torch

B16, F32 = 2.0 ** -8, 2.0 ** -24
INF = float("inf")


def slot_of(table, n_page, page_size, b, s):
    """(page, place) or None where the slot is not there."""
    if s < 0 or s // page_size >= table.shape[1]:
        return None
    page = int(table[b, s // page_size])
    return (page, s % page_size) if 0 <= page < n_page else None


def turned(x, pos, freq, pairs, half):
    """x float64 [T, heads, dh] -> (the columns turned, bound of a float32 kernel; half: its result is bfloat16)."""
    n = len(freq)
    angle = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    c, s = np.cos(angle), np.sin(angle)
    y, size = x.copy(), np.zeros_like(x)
    at = (slice(0, n), slice(n, 2 * n)) if pairs == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size[..., at[0]] = size[..., at[1]] = np.abs(a) + np.abs(b)
    # cos and sin: the reduced angle is rounded to float32 (|r| <= pi: 2^-24 pi of it) and 2 units of the function; the product's rounding in 64 bits
    # moves the angle by 2^-53 of itself; two products and a sum
    far = 2.0 ** -52 * np.abs(angle).max(initial=0.0)
    return y, (3.15 + 4 + 3) * F32 * size + 2 * far * size + (B16 if half else F32) * np.abs(y) * (size > 0) + (B16 if half else 0.0) * np.abs(y) * (size == 0)


def attend(keys, values, table, lens, first, visible, q, scale, half, single=False):
    """keys, values [n_page, KVH, page, dh], q [T, H, dh]: torch tensors; -> (y, bound, rows of a sequence), float64 on the CPU.
    half: the bfloat16 mode."""
    n_page, KVH, page, dh = keys.shape
    T, H = q.shape[:2]
    table, lens, first = table.cpu().numpy(), lens.cpu().tolist(), first.cpu().tolist()
    see = None if visible is None else visible.cpu().numpy().view(np.uint64)
    y, bound, mine = torch.zeros(T, H, dh, dtype=torch.float64), torch.zeros(T, H, dh, dtype=torch.float64), torch.zeros(T, dtype=torch.bool)
    for b, l in enumerate(lens):
        n = first[b + 1] - first[b]
        if n == 0:
            continue
        at = [slot_of(table, n_page, page, b, s) for s in range(l + n)]
        there = torch.tensor([a is not None for a in at], dtype=torch.bool)
        pages, place = torch.tensor([a[0] if a else 0 for a in at]), torch.tensor([a[1] if a else 0 for a in at])
        k, v = (t[pages.to(t.device), :, place.to(t.device)].double().cpu().permute(1, 0, 2) for t in (keys, values))   # [KVH, slots, dh]
        rows = slice(first[b], first[b + 1])
        mine[rows] = True
        seen = torch.zeros(n, l + n, dtype=torch.bool)
        seen[:, :l] = True
        for i in range(n):
            for j in range(n):
                seen[i, l + j] = j <= i if see is None else j < 64 * see.shape[1] and bool(int(see[first[b] + i, j // 64]) >> (j % 64) & 1)
        seen &= there
        if l + n == 0:
            continue
        for h in range(H):
            kk, vv, qq = k[h // (H // KVH)], v[h // (H // KVH)], q[rows, h].double().cpu()
            kk, vv = torch.where(there[:, None], kk, 0.0), torch.where(there[:, None], vv, 0.0)
            s = torch.zeros(n, l + n, dtype=torch.float64)
            for i in range(n):                           # (row by row: what a row does not see is not part of its sums)
                s[i, seen[i]] = scale * (kk[seen[i]] @ qq[i])
            ds = torch.where(seen, abs(scale) * (dh + 6) * F32 * (qq.abs() @ kk.abs().T), 0.0)
            s = torch.where(seen, s, -INF)
            top = s.amax(dim=1, keepdim=True)
            dead = top == -INF
            p = torch.where(s > -INF, torch.exp(s - torch.where(dead, 0.0, top)), 0.0)
            # a weight: its score's and the maximum's error (twice the largest), the argument's roundings, the exponential's, rescalings
            worst = ds.amax(dim=1, keepdim=True)
            span = torch.where(s > -INF, (s.abs() + top.abs()), 0.0)
            e = torch.where(p > 0, ds + worst + 4 * F32 * span + 16 * F32, 0.0)
            e = torch.where(torch.isfinite(e), e, 0.0)
            total = p.sum(dim=1, keepdim=True)
            for i in range(n):
                if dead[i]:
                    continue
                w = p[i, seen[i]]
                out = (w[:, None] * vv[seen[i]]).sum(0) / total[i]
                size = (w[:, None] * vv[seen[i]].abs()).sum(0) / total[i]
                wrong = (w[:, None] * e[i, seen[i]][:, None] * vv[seen[i]].abs()).sum(0) / total[i] + size * (w * e[i, seen[i]]).sum() / total[i]
                count = int(seen[i].sum())
                lost = (B16 if single else 2.0 ** -16 if half else 0.0) + (2 * count + 16) * F32
                y[first[b] + i, h] = out
                bound[first[b] + i, h] = wrong + lost * size + (B16 if half else F32) * (out.abs() + wrong + lost * size) + 1e-38
    return y, bound, mine


def adjust(logits, first, kw, half):
    """logits [T, V] numpy float64 and the arrays of the call as numpy (None: not given) -> (out, bound)."""
    T, V = logits.shape
    out, size = logits.copy(), np.abs(logits)
    get = kw.get
    for t in range(T):
        b, f0, f1 = t, t, t + 1
        if first is not None:
            b = next((i for i in range(len(first) - 1) if first[i] <= t < first[i + 1]), -1)
            if b >= 0:
                f0, f1 = first[b], min(first[b + 1], T)
        x = out[t]
        if b >= 0:
            times, asked = np.zeros(V, np.int64), np.zeros(V, bool)
            if get("tokens") is not None:
                row = get("tokens")[b]
                n = len(row) if get("n_token") is None else min(int(get("n_token")[b]), len(row))
                m = 0 if get("n_prompt") is None else int(get("n_prompt")[b])
                for i in range(n):
                    if 0 <= row[i] < V:
                        if i < m:
                            asked[row[i]] = True
                        else:
                            times[row[i]] += 1
            if get("draft") is not None:
                for j in range(f1 - f0):
                    see = get("visible")
                    ok = f0 + j <= t if see is None else j < 64 * see.shape[1] and bool(int(see[t, j // 64]) >> (j % 64) & 1)
                    v = get("draft")[f0 + j]
                    if ok and 0 <= v < V:
                        times[v] += 1
            met = asked | (times > 0)
            if get("repetition") is not None:
                r = float(get("repetition")[b])
                x[met] = np.where(x[met] > 0, x[met] / r, x[met] * r)
                size[t] = np.maximum(size[t], np.abs(x))
            gen = times > 0
            if get("frequency") is not None:
                x[gen] -= float(get("frequency")[b]) * times[gen]
                size[t][gen] += abs(float(get("frequency")[b])) * times[gen]
            if get("presence") is not None:
                x[gen] -= float(get("presence")[b])
                size[t][gen] += abs(float(get("presence")[b]))
            if get("bias") is not None:
                last = {int(v): float(a) for v, a in zip(get("bias_ids")[b], get("bias")[b]) if 0 <= v < V}
                for v, a in last.items():
                    x[v] += a
                    size[t][v] += abs(a)
        if get("mask") is not None:
            row = t if get("mask_row") is None else int(get("mask_row")[t])
            if 0 <= row < len(get("mask")):
                word = get("mask")[row].view(np.uint32)
                allowed = (word[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
                x[allowed == 0] = -INF
    with np.errstate(invalid="ignore"):
        changed = 6 * F32 * size
        bound = np.where(out == logits, 0.0, changed + (B16 if half else 0.0) * (np.abs(out) + changed) + 1e-38)
    return out, bound


def keep(store, table, lens, first, path, n_keep):
    """store numpy [layers, pages, KVH, page, dh] -> a copy after the move."""
    out = store.copy()
    n_page, page = store.shape[1], store.shape[3]
    for b in range(len(lens)):
        n = first[b + 1] - first[b]
        for j in range(min(int(n_keep[b]), path.shape[1])):
            i = int(path[b, j])
            if i < j or i >= n:
                continue
            a, c = slot_of(table, n_page, page, b, lens[b] + i), slot_of(table, n_page, page, b, lens[b] + j)
            if a and c:
                out[:, c[0], :, c[1]] = store[:, a[0], :, a[1]]
    return out
