"""CPU reference in float64 for the operators of a step that answers a batch of requests over one paged cache: written from the
definitions, one sequence, token and row at a time, for tests only."""
import numpy as np

MOST = 1 << 30


def page_tables(cached, new, table, free_pages, free_at, page, n_pages, n_tokens, offset=None):
    """(table, first, length, position, slot, taken) as lists; table a list of lists, copied"""
    table = [list(r) for r in table]
    first, length, position, slot, taken = [0], [], [], [], 0
    for s, c in enumerate(cached):
        c = min(max(c, 0), MOST)
        n = min(max(new[s], 0), n_tokens - first[-1])
        first.append(first[-1] + n)
        length.append(min(c + n, MOST))
        width = len(table[s])
        for j in range(-(-c // page), -(-length[s] // page)):
            if j >= width:
                break
            at = free_at + taken
            number = free_pages[at] if 0 <= at < len(free_pages) else -1
            table[s][j] = number if 0 <= number < n_pages else -1
            taken += 1
        for j in range(c, c + n):
            number = table[s][j // page] if j // page < width and j < MOST else -1
            position.append((offset[s] if offset else 0) + j)
            slot.append(number * page + j % page if 0 <= number < n_pages else -1)
    return table, first, length, position, slot, taken


def rows_of(pages, table, n):
    """Rows of the first n positions of one table's row and which of them there are: pages [n_pages, heads, page, d] -> [heads, n, d], [n]"""
    at = np.arange(n)
    number = np.asarray(table, dtype=np.int64)[at // pages.shape[2]] if n else np.zeros(0, np.int64)
    there = (number >= 0) & (number < pages.shape[0])
    return pages[np.where(there, number, 0), :, at % pages.shape[2]].transpose(1, 0, 2), there


def attention(q, k, v, there, before, scale):
    """One sequence: q [t, hq, d], k, v [hk, positions, d], of which token i sees the first before + i + 1 that are there; [t, hq, d]"""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    t, hq, d = q.shape
    group = hq // k.shape[0]
    out = np.zeros((t, hq, d))
    for i in range(t):
        see = np.flatnonzero(there[:max(0, before + i + 1)])
        if len(see) == 0:
            continue
        for h in range(hq):
            z = k[h // group][see] @ q[i, h] * scale
            w = np.exp(z - z.max())
            out[i, h] = (w / w.sum()) @ v[h // group][see]
    return out


def order(logits):
    """Logits as they count (nan: -inf, +inf: the largest finite number), and the indices in order: larger first, the lower index first"""
    x = np.asarray(logits, dtype=np.float64)
    x = np.minimum(np.where(np.isnan(x), -np.inf, x), float(np.finfo(np.float32).max))
    return x, np.argsort(-x, kind="stable")


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The order, its running sums of weights, and how many entries are kept"""
    x, at = order(logits)
    there = int((x > -np.inf).sum())
    if there == 0:
        return at, np.zeros(len(x)), 0
    z = x[at[:there]] - x[at[0]]
    if not temperature > 0:
        return at, np.ones(1), 1
    w = np.exp(z / float(temperature))
    total = np.cumsum(w)
    most = there if not top_k > 0 else min(int(top_k), there)
    n = most
    if top_p < 1:
        n = min(n, int(np.searchsorted(total[:most], float(top_p) * total[most - 1], side="left")) + 1)
    if min_p > 0:
        n = min(n, int((w >= float(min_p)).sum()))
    return at, total, max(1, n)


def sample(logits, u, **settings):
    """(token, kept)"""
    at, total, n = kept(logits, **settings)
    if n == 0:
        return -1, 0
    r = int(np.searchsorted(total[:n], float(u) * total[n - 1], side="right"))
    return int(at[min(r, n - 1)]), n
