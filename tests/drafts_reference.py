"""The drafting operators' definitions in 64 bits (angles in 80), token by token, for the tests."""
import math

import numpy as np
import torch


def turned(x, positions, freqs, interleaved, amplitude=1.0):
    """x [rows, heads, d] (any type) turned to `positions` -> fp64, and |a| + |b| of every channel's pair, by which errors are measured."""
    y = x.detach().cpu().double().numpy().copy()
    size = np.abs(y)
    f = np.asarray(freqs.cpu() if hasattr(freqs, "cpu") else freqs, dtype=np.longdouble)
    n = len(f)
    a, b = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * f
    c, s = (amplitude * t(angle).astype(np.float64)[:, None] for t in (np.cos, np.sin))
    u, v = y[..., a].copy(), y[..., b].copy()
    size[..., a] = size[..., b] = abs(amplitude) * (np.abs(u) + np.abs(v))
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return torch.from_numpy(y), torch.from_numpy(size)


def random_tree(n, r, depth=8, branch=4, forest=False):
    """Parents of n tokens, earlier ones each."""
    parents, level, children = [-1], [0], [0]
    for i in range(1, n):
        room = [k for k in range(i) if level[k] < depth and children[k] < branch] or [i - 1]
        p = -1 if forest and r.random() < 0.2 else r.choice(room)
        parents.append(p)
        level.append(0 if p < 0 else level[p] + 1)
        children.append(0)
        if p >= 0:
            children[p] += 1
    return parents[:n], level[:n]


def seen_by(parents, n, held):
    """[n, held]: which of the tokens held a query of the tree, whose tokens are the last n, sees."""
    seen = torch.zeros(n, held, dtype=torch.bool)
    seen[:, :max(held - n, 0)] = True
    for i in range(n):
        at = i
        while at >= 0:
            if held - n + at >= 0:
                seen[i, held - n + at] = True
            at = parents[at] if -1 <= parents[at] < at else -1
    return seen


def attend(q, k, v, scale, seen):
    """q [nq, H, d], k, v [nk, Hkv, d], seen [nq, nk] -> out, size, lse as serving_reference.attend."""
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    (nq, H, d), G = q.shape, q.shape[1] // max(k.shape[1], 1)
    out, size, lse = torch.zeros(nq, H, d, dtype=torch.float64), torch.zeros(nq, H, d, dtype=torch.float64), torch.full((nq, H), -math.inf, dtype=torch.float64)
    some = seen.any(-1)
    for h in range(k.shape[1]):
        for g in range(h * G, (h + 1) * G):
            s = (scale * (q[:, g] @ k[:, h].T)).masked_fill(~seen, -math.inf)
            top = torch.where(some, s.amax(-1), 0.0) if s.shape[1] else torch.zeros(nq, dtype=torch.float64)
            w = torch.exp(s - top[:, None])
            total = w.sum(-1)
            by = torch.where(total > 0, total, 1.0)[:, None]
            out[:, g], size[:, g] = w @ v[:, h] / by, w @ v[:, h].abs() / by
            lse[:, g] = torch.where(some, top + total.log(), -math.inf)
    return out, size, lse


def _softmax(x, T):
    x = x.double().numpy() / T
    if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
        return None
    w = np.exp(x - x.max())
    return w / w.sum()


def verify(logits, drafts, tokens, parents, uniform, T, distinct):
    """One sequence (CPU tensors, lists) -> path, accepted, next, margin: how near, relative, the nearest decision was to its border."""
    n, V = len(parents), logits.shape[1] if logits.dim() == 2 else 0
    path, node, margin = [0], 0, math.inf
    while True:
        children = [i for i in range(node + 1, n) if parents[i] == node and 0 <= tokens[i] < V]
        row = logits[node]
        if T == 0:
            x = row.double().numpy()
            if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
                return path, len(path) - 1, -1, margin
            best = int(np.argmax(x))
            taken = next((i for i in children if tokens[i] == best), None)
            if taken is None:
                return path, len(path) - 1, best, margin
            path.append(taken)
            node = taken
            continue
        p = _softmax(row, T)
        leaf = not any(parents[i] == node for i in range(node + 1, n))
        q = _softmax(drafts[node], T) if drafts is not None and not leaf else None
        if p is None or (drafts is not None and not leaf and q is None):
            return path, len(path) - 1, -1, margin
        w, q0, taken, tried = p.copy(), q, None, []
        for i in children:
            x = tokens[i]
            if (distinct or drafts is None) and x in tried:
                continue
            qx = 1.0 if drafts is None else q[x]
            left, right = float(uniform[i]) * qx * w.sum(), w[x]
            if left > 0 or right > 0:            # (zero against zero is no border: refused)
                margin = min(margin, abs(left - right) / max(left, right))
            if left < right:
                taken = i
                break
            tried.append(x)
            one = np.zeros(V)
            one[x] = 1
            w = np.maximum(w / w.sum() - (one if drafts is None else q), 0) if drafts is not None else w * (1 - one)
            if drafts is not None and distinct:
                q = q0.copy()
                q[tried] = 0
                q = q / q.sum() if q.sum() > 0 else q
            if not w.sum() > 1e-13:              # (nothing but roundings is left, by definition)
                w = p.copy()
                break
        if taken is not None:
            path.append(taken)
            node = taken
            continue
        if not w.sum() > 0:
            w = p.copy()
        sums = np.cumsum(w)
        target = float(uniform[0]) * sums[-1]
        margin = min(margin, np.abs(sums - target).min() / sums[-1] * len(sums))
        return path, len(path) - 1, int(np.argmax(sums > target)), margin


def byte_places(page_size, Hkv, d, head, in_page):
    """Bytes of a page that a token owns in one head, in a fixed order."""
    G, base, t = d // 32, (head * (page_size // 16) + in_page // 16) * 20 * d, in_page % 16
    at = list(range(base + t * d // 2, base + (t + 1) * d // 2)) + list(range(base + 8 * d + 4 * G * t, base + 8 * d + 4 * G * (t + 1)))
    for w in range(8 * G):
        at += [base + 10 * d + t // 2 * d + 4 * w + 2 * (t % 2) + i for i in range(2)]
    for w in range(2 * G):
        at += [base + 18 * d + t // 2 * 8 * G + 4 * w + 2 * (t % 2) + i for i in range(2)]
    return at
