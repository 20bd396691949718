"""The operators of a step that answers a batch of requests over one paged cache, as cases that can be timed and checked one by one.

The cache is a pool of pages of some positions each; a request's positions lie in the pages that its row of a table names.  Requests that
begin with the same text (a system prompt, a document that several questions are about) share the pages of that prefix.  A step's operators:
  tables   which pages and places the step's new tokens get, from the requests' lengths and a list of free pages
  append   the new tokens' keys and values move to their places
  attend   attention of the tokens over their group's prefix and over their own positions
  sample   the next token of every request, from given random numbers: temperature, top-k, top-p, min-p

Keys of a case beside `op` and `type` (element type):
  tables   seqs, tokens (new ones of a sequence, the most), cached (positions of the longest sequence), page (positions of a page), offset
           (positions count from a prefix's end)
  append   tokens, kv_heads, dim, page
  attend   seqs, tokens (new ones of a sequence, the most), q_heads, kv_heads, dim, prefixes (groups of sequences), prefix (positions of the
           longest), length (own positions of the longest sequence, the new ones among them), page, ragged (sequences of several lengths)
  sample   rows, vocab, filters (of k, p, m: which of top-k, top-p and min-p are given), greedy (share of rows without sampling)
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}


def _tables(name=None, seqs=1, tokens=1, cached=1000, page=16, offset=True):
    c = dict(op="tables", seqs=seqs, tokens=tokens, cached=cached, page=page, offset=offset)
    return dict(c, name=name) if name else c


def _append(name=None, tokens=1, kv_heads=8, dim=128, page=16, type="f16"):
    c = dict(op="append", tokens=tokens, kv_heads=kv_heads, dim=dim, page=page, type=type)
    return dict(c, name=name) if name else c


def _attend(name=None, seqs=1, tokens=1, q_heads=32, kv_heads=8, dim=128, prefixes=1, prefix=1000, length=1000, page=16, ragged=True, type="f16"):
    c = dict(op="attend", seqs=seqs, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim, prefixes=prefixes, prefix=prefix, length=length,
             page=page, ragged=ragged, type=type)
    return dict(c, name=name) if name else c


def _sample(name=None, rows=1, vocab=128256, filters="kp", greedy=0.0, type="f16"):
    c = dict(op="sample", rows=rows, vocab=vocab, filters=filters, greedy=greedy, type=type)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of 64 requests, a token each (launch latency)
        _tables("tables_64", 64, 1, 1000, 16, True),
        # a step that takes in the prompts of many requests beside decoding others
        _tables("tables_1000_prompts", 1000, 130, 300, 16, False),
        # the rows of a decode step of 64 requests, 8 kv heads (launch latency)
        _append("append_64", 64),
        # the rows of the largest prompt chunk of the tier table
        _append("append_16384", 16384, 8, 128, 64, "bf16"),
        # three short requests behind a short common prompt in the heads of the tests' miniature (launch latency)
        _attend("attend_3", 3, 1, 4, 2, 128, 1, 77, 40, 16),
        # 64 requests about one long document in the 8B-shaped stack's heads
        _attend("attend_64_one_document", 64, 1, 32, 8, 128, 1, 32761, 1000, 16),
        # requests of several lengths that share nothing, heads of 64
        _attend("attend_48_ragged", 48, 1, 16, 8, 64, 0, 0, 8190, 64, True, "bf16"),
        # a large batch behind four system prompts, the MoE stack's heads, a drafted token beside the last one
        _attend("attend_256_four_prompts", 256, 2, 32, 4, 128, 4, 4093, 2000, 32, True, "bf16"),
        # the prompts of eight new requests behind a common system prompt
        _attend("attend_8_prompts", 8, 512, 32, 8, 128, 1, 2048, 512, 128),
        # one request with a small vocabulary (launch latency)
        _sample("sample_1", 1, 32000, "kp"),
        # a batch of requests with settings of their own; a part of them does not sample
        _sample("sample_16", 16, 128256, "kpm", 0.25, "bf16"),
        # a large batch, fp32 logits, top-p alone
        _sample("sample_256", 256, 128256, "p", 0.0, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "attend", "sample", "sample", "sample"])
    page = rng.choice([16, 32, 64, 128])
    if op == "tables":
        seqs = _log(rng, 1, 1000)
        return _tables(None, seqs, _log(rng, 1, min(4096, 130000 // seqs)), _log(rng, 1, 8000), page, rng.random() < 0.5)
    kv, dim = rng.choice([2, 4, 8]), rng.choice([64, 128])
    if op == "append":
        return _append(None, _log(rng, 1, 16384), kv, dim, page, rng.choice(["f16", "bf16"]))
    if op == "attend":
        q = kv * rng.choice([1, 2, 4, 8])
        seqs = _log(rng, 1, 256)
        tokens = 1 if rng.random() < 0.5 else _log(rng, 1, 512)
        most = min(8190, 700000000 // (seqs * kv * dim * 4), 140000000000 // (4 * seqs * tokens * q * dim))
        length = _log(rng, 1, max(2, most))
        tokens = min(tokens, length)
        prefixes = rng.choice([0, 1, 1, 2, 5])
        most = min(33000, 140000000000 // (4 * seqs * tokens * q * dim) - length)
        prefix = _log(rng, 1, max(2, most)) if prefixes else 0
        return _attend(None, seqs, tokens, q, kv, dim, min(prefixes, seqs), prefix, length, page, rng.random() < 0.7, rng.choice(["f16", "bf16"]))
    rows = _log(rng, 1, 256)
    return _sample(None, rows, _log(rng, 1000, 128256), rng.choice(["", "k", "p", "m", "kp", "kpm"]), rng.choice([0.0, 0.0, 0.5]),
                   rng.choice(["f16", "bf16", "f32"]))


# ------------------------------------------------------------------ sizes that a case fixes

def _sizes(case):
    """New tokens of each sequence: the most, and where there are several sequences also fewer."""
    t = case["tokens"]
    return [t - (5 * i) % max(1, (t + 1) // 2) for i in range(case["seqs"])]


def _lengths(case):
    """Own positions of each sequence behind the step."""
    c, s = case["length"], case["seqs"]
    return [max(t, c if not case["ragged"] else c - (i * i * c) // (s * s)) for i, t in enumerate(_sizes(case))]


def _cached(case):
    c, s = case["cached"], case["seqs"]
    return [(c * (i + 1)) // s if i % 7 != 3 else 0 for i in range(s)]


def _groups(case):
    """First sequence of each prefix's group; with several prefixes an eighth of the sequences, the last ones, stand behind none."""
    p, s = case["prefixes"], case["seqs"]
    return [i * s if p < 2 else i * s * 7 // (8 * p) for i in range(p + 1)]


def _prefixes(case):
    return [max(1, case["prefix"] - 37 * i) for i in range(case["prefixes"])]


def work(case):
    if case["op"] == "tables":
        return {"bytes": 4.0 * (3 * case["seqs"] + 2 * case["seqs"] + 2 * sum(_sizes(case)) + 2 * sum(_sizes(case)) / case["page"]), "flops": 0.0}
    e = BYTES[case["type"]]
    if case["op"] == "append":
        return {"bytes": 4.0 * case["tokens"] * case["kv_heads"] * case["dim"] * e, "flops": 0.0}
    if case["op"] == "sample":
        return {"bytes": float(case["rows"] * case["vocab"] * e), "flops": 4.0 * case["rows"] * case["vocab"]}
    d, hq, hk = case["dim"], case["q_heads"], case["kv_heads"]
    ts, ls, gs, ps = _sizes(case), _lengths(case), _groups(case), _prefixes(case)
    rows = 2 * hk * (sum(ls) + sum(ps)) + 2 * hq * sum(ts)
    seen = sum(t * l - t * (t - 1) // 2 for t, l in zip(ts, ls)) + sum(p * sum(ts[gs[i]:gs[i + 1]]) for i, p in enumerate(ps))
    return {"bytes": float(rows * d * e), "flops": 4.0 * d * hq * seen}


# ------------------------------------------------------------------ inputs

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _deal(rows, page, g, spare=0):
    """Pages for rows of some positions each, in no order: the table [rows, widest], -1 behind a row's last page, and the pages left over."""
    need = [(n + page - 1) // page for n in rows]
    order = torch.randperm(sum(need) + spare, generator=g, device=DEVICE).to(torch.int32)
    width = max(need + [1])
    count = torch.tensor(need, device=DEVICE, dtype=torch.int64)
    at = (count.cumsum(0) - count)[:, None] + torch.arange(width, device=DEVICE)
    table = torch.where(torch.arange(width, device=DEVICE) < count[:, None], order[at.clamp(max=order.numel() - 1)], -1)
    return table.contiguous(), order[sum(need):].contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "tables":
        ts, cs, page = _sizes(case), _cached(case), case["page"]
        s["cached"], s["new"], s["n"] = _ints(cs), _ints(ts), sum(ts)
        more = sum((c + t + page - 1) // page - (c + page - 1) // page for c, t in zip(cs, ts))
        table, s["free"] = _deal(cs, page, g, more + 50)
        width = (case["cached"] + case["tokens"] + page - 1) // page + 1
        s["table"] = torch.full((case["seqs"], max(width, table.shape[1])), -1, dtype=torch.int32, device=DEVICE)
        s["table"][:, :table.shape[1]] = table
        s["pages"] = sum((c + page - 1) // page for c in cs) + more + 50
        s["free_at"] = torch.randint(0, 50, (1,), generator=g, device=DEVICE).to(torch.int32)
        s["offset"] = torch.randint(0, 4000, (case["seqs"],), generator=g, device=DEVICE).to(torch.int32) if case["offset"] else None
        return s
    dt = TYPES[case["type"]]
    if case["op"] == "append":
        n, h, d, page = case["tokens"], case["kv_heads"], case["dim"], case["page"]
        qkv = _normal(g, n, 6 * h * d).to(dt)                       # the rows that a QKV projection leaves, four query heads a kv head
        s["k"], s["v"] = qkv[:, 4 * h * d:5 * h * d].view(n, h, d), qkv[:, 5 * h * d:].view(n, h, d)
        pages = n // page * 3 // 2 + 4 + (n if n <= 256 else 0)
        pool = _normal(g, pages, 2, h, page, d).to(dt)
        s["k_pages"], s["v_pages"] = pool[:, 0], pool[:, 1]
        if n <= 256:        # decoding: every row to a page of its own
            s["slot"] = torch.randperm(pages, generator=g, device=DEVICE)[:n] * page + torch.randint(0, page, (n,), generator=g, device=DEVICE)
        else:               # prompts: runs of rows in pages that lie in no order
            full = (n + page - 1) // page
            s["slot"] = (torch.randperm(pages, generator=g, device=DEVICE)[:full, None] * page + torch.arange(page, device=DEVICE)).flatten()[:n]
        s["slot"] = s["slot"].to(torch.int32)
        return s
    if case["op"] == "sample":
        n, v = case["rows"], case["vocab"]
        s["logits"] = (_normal(g, n, v) * 2.5).to(dt)
        s["u"] = torch.rand(n, generator=g, device=DEVICE)
        i = torch.arange(n, device=DEVICE)
        s["temperature"] = torch.where(i < round(case["greedy"] * n), 0.0, torch.tensor([0.7, 1.0, 0.9, 1.3], device=DEVICE)[i % 4]).float()
        s["top_k"] = _ints([50, 0, 20, 1000, 1]).repeat(n // 5 + 1)[:n].contiguous() if "k" in case["filters"] else None
        s["top_p"] = torch.tensor([0.9, 0.95, 1.0], device=DEVICE).repeat(n // 3 + 1)[:n].contiguous() if "p" in case["filters"] else None
        s["min_p"] = torch.tensor([0.05, 0.0], device=DEVICE).repeat(n // 2 + 1)[:n].contiguous() if "m" in case["filters"] else None
        return s
    ts, ls, gs, ps = _sizes(case), _lengths(case), _groups(case), _prefixes(case)
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    first = [sum(ts[:i]) for i in range(len(ts) + 1)]
    n = first[-1]
    s["first"], s["length"], s["sizes"] = _ints(first), _ints(ls), (ts, ls, gs, ps, first)
    table, _ = _deal(ls + ps, page, g)
    s["table"], s["prefix_table"] = table[:len(ls), :(max(ls) + page - 1) // page], table[len(ls):]
    s["group_first"] = _ints(gs) if ps else None
    s["prefix_length"] = _ints(ps) if ps else None
    s["q"] = (_normal(g, n, (hq + 2 * hk) * d) * 2).to(dt)[:, :hq * d].view(n, hq, d)
    pages = sum((x + page - 1) // page for x in ls + ps)
    pool = torch.empty(pages, 2, hk, page, d, dtype=dt, device=DEVICE)
    for i in range(0, pages, 4096):
        pool[i:i + 4096] = _normal(g, *pool[i:i + 4096].shape)
    s["k_pages"], s["v_pages"] = pool[:, 0], pool[:, 1]
    # where each token lies among its sequence's: for the plain form, which works on padded sequences
    s["seq"] = torch.repeat_interleave(torch.arange(len(ts), device=DEVICE), torch.tensor(ts, device=DEVICE))
    s["number"] = torch.arange(n, device=DEVICE) - s["first"][s["seq"]]
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        from paper_2604_26334_amd import binding as B
        if case["op"] == "tables":
            return (s["table"],) + B.page_tables(s["cached"], s["new"], s["table"], s["free"], s["free_at"], page=case["page"], n_pages=s["pages"],
                                                 n_tokens=s["n"], offset=s["offset"])
        if case["op"] == "append":
            return B.page_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slot"])
        if case["op"] == "sample":
            return B.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return B.page_attention(s["q"], s["k_pages"], s["v_pages"], s["first"], s["length"], s["table"], max_length=max(s["sizes"][1]),
                                max_tokens=case["tokens"], group_first=s["group_first"], prefix_length=s["prefix_length"],
                                prefix_table=s["prefix_table"] if case["prefixes"] else None, max_prefix=case["prefix"])
    return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[case["op"]](s)


def _plain_tables(s):
    page, table = s["case"]["page"], s["table"]
    cached, new = s["cached"].long(), s["new"].long()
    first = torch.cat((new.new_zeros(1), new.cumsum(0)))
    length = cached + new
    held, full = (cached + page - 1) // page, (length + page - 1) // page
    more = full - held
    before = more.cumsum(0) - more
    entry = torch.arange(table.shape[1], device=DEVICE)
    fresh = (entry >= held[:, None]) & (entry < full[:, None])
    at = s["free_at"].long() + before[:, None] + entry - held[:, None]
    table.copy_(torch.where(fresh, s["free"][at.clamp(0, s["free"].numel() - 1)], table))
    seq = torch.searchsorted(first, torch.arange(s["n"], device=DEVICE), right=True) - 1
    place = cached[seq] + torch.arange(s["n"], device=DEVICE) - first[seq]
    position = place + (s["offset"].long()[seq] if s["offset"] is not None else 0)
    slot = table[seq, place // page] * page + place % page
    return table, first.int(), length.int(), position.int(), slot.int(), more.sum(0, keepdim=True).int()


def _plain_append(s):
    page = s["case"]["page"]
    slot = s["slot"].long()
    s["k_pages"][slot // page, :, slot % page] = s["k"]
    s["v_pages"][slot // page, :, slot % page] = s["v"]
    return s["k_pages"], s["v_pages"]


def _rows_of(pages, table, n):
    """The first n positions that tables [rows, width] name: [rows, heads, n, dim], in 32 bits"""
    x = pages[table.long().clamp(min=0)].float()                    # [rows, width, heads, page, dim]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :n]


def _part(q, k, v, seen):
    """Unscaled sums of one part of the positions: largest score, weights' sum, weighted values"""
    z = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(q.shape[-1]))
    if seen is not None:
        z.masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    w = (z - torch.where(m > -math.inf, m, 0.0)).exp_()
    return m, w.sum(-1, keepdim=True), torch.matmul(w, v)


def _plain_attend(s):
    case = s["case"]
    ts, ls, gs, ps, first = s["sizes"]
    b, t, n, hq, hk, d = case["seqs"], max(ts), first[-1], case["q_heads"], case["kv_heads"], case["dim"]
    group = hq // hk
    q = s["q"].float()
    # own positions, on padded sequences; token i of a sequence sees length - tokens + i + 1 of them
    x = q.new_zeros(b, t, hq, d)
    x[s["seq"], s["number"]] = q
    x = x.view(b, t, hk, group, d).permute(0, 2, 3, 1, 4).reshape(b, hk, group * t, d)
    limit = (s["length"] - (s["first"][1:] - s["first"][:-1]))[:, None] + torch.arange(t, device=DEVICE) + 1
    seen = torch.arange(max(ls), device=DEVICE) < limit[:, None, None, :, None]
    seen = seen.expand(b, 1, group, t, max(ls)).reshape(b, 1, group * t, max(ls))
    part = _part(x, _rows_of(s["k_pages"], s["table"], max(ls)), _rows_of(s["v_pages"], s["table"], max(ls)), seen)
    back = [p.view(b, hk, group, t, -1).permute(0, 3, 1, 2, 4).reshape(b, t, hq, -1)[s["seq"], s["number"]] for p in part]
    m1, l1, o1 = back
    # each prefix once, for all tokens of its group
    m2, l2, o2 = torch.full_like(m1, -math.inf), torch.zeros_like(l1), torch.zeros_like(o1)
    for i, p in enumerate(ps):
        rows = slice(first[gs[i]], first[gs[i + 1]])
        x = q[rows].view(-1, hk, group, d).permute(1, 2, 0, 3).reshape(hk, -1, d)
        k, v = (_rows_of(s[name], s["prefix_table"][i:i + 1], p)[0] for name in ("k_pages", "v_pages"))
        m, l, o = (y.view(hk, group, -1, y.shape[-1]).permute(2, 0, 1, 3).reshape(-1, hq, y.shape[-1]) for y in _part(x, k, v, None))
        m2[rows], l2[rows], o2[rows] = m, l, o
    top = torch.maximum(m1, m2)
    f1, f2 = (m1 - top).exp(), (m2 - top).exp()
    return ((o1 * f1 + o2 * f2) / (l1 * f1 + l2 * f2)).to(s["q"].dtype)


def _plain_sample(s):
    logits = s["logits"]
    v = logits.shape[1]
    order = torch.sort(logits, dim=-1, descending=True, stable=True).indices          # equal logits: the lowest index first
    x = logits.gather(1, order).double()
    temp = s["temperature"][:, None].double()
    w = ((x - x[:, :1]) / torch.where(temp > 0, temp, 1.0)).exp()                 # 64 bits: a border of the running sum lies among many
    run_sum = w.cumsum(-1)
    most = torch.full_like(order[:, :1], v)
    if s["top_k"] is not None:
        k = s["top_k"][:, None].long()
        most = torch.where((k > 0) & (k < v), k, v)
    n = most
    if s["top_p"] is not None:
        p = s["top_p"][:, None].double()
        goal = p * run_sum.gather(1, most - 1)
        n = torch.where(p < 1, torch.minimum(n, (run_sum < goal).sum(-1, keepdim=True) + 1), n)
    if s["min_p"] is not None:
        n = torch.minimum(n, (w >= s["min_p"][:, None].double()).sum(-1, keepdim=True))
    n = torch.where(temp > 0, n, 1).clamp(min=1)
    at = (run_sum <= s["u"][:, None].double() * run_sum.gather(1, n - 1)).sum(-1, keepdim=True)
    token = order.gather(1, torch.minimum(at, n - 1))
    return token[:, 0].int(), n[:, 0].int()


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    if case["op"] in ("tables", "sample"):
        return None          # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        if s["k_pages"].numel() > 1 << 26:
            return None
        out = []
        for x, pages in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
            y = pages.transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"]).double()
            y.index_copy_(0, s["slot"].long(), x.double())
            out.append(y.view(-1, case["page"], case["kv_heads"], case["dim"]).transpose(1, 2).contiguous())
        return tuple(out)
    if work(case)["flops"] > 4e11:
        return None
    ts, ls, gs, ps, first = s["sizes"]
    group, page = case["q_heads"] // case["kv_heads"], case["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)

    def rows(pages, table, n, h):
        at = torch.arange(n, device=DEVICE)
        return pages[table[at // page].long(), h, at % page].double()
    for h in range(case["kv_heads"]):
        heads = slice(h * group, (h + 1) * group)
        shared = [[rows(s[x], s["prefix_table"][i], p, h) for x in ("k_pages", "v_pages")] for i, p in enumerate(ps)]
        for b, (t, l) in enumerate(zip(ts, ls)):
            k, v = (rows(s[x], s["table"][b], l, h) for x in ("k_pages", "v_pages"))
            p = 0
            for i in range(len(ps)):
                if gs[i] <= b < gs[i + 1]:
                    k, v, p = torch.cat((shared[i][0], k)), torch.cat((shared[i][1], v)), ps[i]
            x = s["q"][first[b]:first[b + 1], heads].double().reshape(-1, case["dim"])
            z = x @ k.T / math.sqrt(case["dim"])
            limit = p + l - t + 1 + torch.arange(t, device=DEVICE).repeat_interleave(group)
            z.masked_fill_(torch.arange(p + l, device=DEVICE) >= limit[:, None], -math.inf)
            out[first[b]:first[b + 1], heads] = (torch.softmax(z, -1) @ v).view(t, group, case["dim"])
    return out
