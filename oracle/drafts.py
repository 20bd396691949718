"""CPU reference in float64 for the operators of a step that answers several drafted tokens: written from the definitions,
row by row, for tests only."""
import math

import numpy as np


def parents_of(parent):
    """Parents as the operators read them: node i's parent lies in 0 .. i - 1, anything else makes it a node without one (-1)."""
    return [int(p) if 0 <= p < i else -1 for i, p in enumerate(parent)]


def qk_norm_rope(x, gain, positions, inv_freq, eps, norm, pairs):
    """x [tokens, heads, dim] float64, gain [dim] or None; inv_freq float32 [rot / 2]"""
    y = np.array(x, dtype=np.float64)
    if norm:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if gain is not None:
            y = y * np.asarray(gain, dtype=np.float64)
    out = y.copy()
    half = len(inv_freq)
    for t, pos in enumerate(positions):
        for i, f in enumerate(inv_freq):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            turn = float(pos) * float(f)
            c, s = math.cos(turn), math.sin(turn)
            out[t, :, a] = y[t, :, a] * c - y[t, :, b] * s
            out[t, :, b] = y[t, :, b] * c + y[t, :, a] * s
    return out


def tree_attention(q, k_new, v_new, k_cache, v_cache, context, parent, scale):
    """One sequence: q [t, hq, d], k_new / v_new [t, hk, d], k_cache / v_cache [hk, cap, d]; float64 result [t, hq, d]"""
    q, k_new, v_new = (np.asarray(a, dtype=np.float64) for a in (q, k_new, v_new))
    t, hq, d = q.shape
    group = hq // k_new.shape[1]
    up = parents_of(parent)
    out = np.zeros((t, hq, d))
    for h in range(k_new.shape[1]):
        kc, vc = (np.asarray(a[h, :context], dtype=np.float64) for a in (k_cache, v_cache))
        for i in range(t):
            line, j = [], i
            while j >= 0:
                line.append(j)
                j = up[j]
            k, v = np.concatenate([kc, k_new[line, h]]), np.concatenate([vc, v_new[line, h]])
            for g in range(group):
                z = k @ q[i, h * group + g] * scale
                w = np.exp(z - z.max())
                out[i, h * group + g] = (w / w.sum()) @ v
    return out


def _row(logits, temperature):
    """Probabilities of a row: nan counts as -inf, +inf as the largest finite number; a row of -inf alone has none (zeros)."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    x = np.minimum(x, np.finfo(np.float32).max)
    m = x.max()
    if m == -np.inf:
        return np.zeros_like(x)
    if not temperature > 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0          # the lowest index among equals
        return p
    with np.errstate(over="ignore"):
        e = np.exp((x - m) / float(temperature))
    return e / e.sum()


def verify_tree(target, token, parent, u_accept, u_sample, draft=None, temperature=1.0, max_children=1 << 30):
    """One sequence: target [t, V], token / parent [t], u_accept [t], u_sample: (path, next token)"""
    t = len(token)
    if t == 0:
        return [], -1
    up = parents_of(parent)
    V = target.shape[1]
    greedy = not temperature > 0
    here, path = 0, [0]
    while True:
        p = _row(target[here], temperature)
        q = None if draft is None or greedy else _row(draft[here], temperature)
        rest, c, w, went = p.copy(), 0.0, 1.0, None
        children = [i for i in range(1, t) if up[i] == here][:max_children]
        for i in children:
            x, u = int(token[i]), float(u_accept[i])
            inside = 0 <= x < V
            if q is None:
                px = rest[x] if inside else 0.0
                if px > u * w:
                    went = i
                    break
                if inside and not greedy:
                    rest[x] = 0.0
                    w = rest.sum()
            else:
                if (p[x] if inside else 0.0) > (c + u * w) * (q[x] if inside else 0.0):
                    went = i
                    break
                c += w
                rest = np.maximum(p - c * q, 0.0)
                w = rest.sum()
        if went is None:
            break
        here = went
        path.append(here)
    if rest.sum() <= 0:      # nothing left to draw from: the target's own row
        rest = p
    if rest.sum() <= 0:
        return path, -1
    run = np.cumsum(rest)
    over = np.nonzero(run > float(u_sample) * run[-1])[0]
    return path, int(over[0] if len(over) else np.nonzero(rest)[0][-1])
