"""The operators of a step that answers several drafted tokens at once, as cases that can be timed and checked one by one.

A step of that kind runs a tree of drafted tokens (node 0 is the last known token, every other node a draft that follows
its parent) through the stack in one forward.  Its operators:
  rope     norms of queries and keys for each head, with the position rotation in the same pass
  tree     attention of the tree's tokens over the cache and over their own ancestors
  verify   which drafts the target's logits accept from given random numbers, and the token behind the last accepted one
  keep     the accepted tokens' rows of the cache move to the places behind the context

Keys of a case beside `op` and `type` (element type):
  rope     tokens, q_heads, kv_heads, dim, rot (rotated dimensions), pairs (neighbours instead of halves), norm
  tree     seqs, tokens (of the largest tree), branch (children of a node; 1: a chain), q_heads, kv_heads, dim, context (of the
           longest sequence), ragged (sequences of several lengths)
  verify   seqs, tokens, branch, vocab, drafts (the drafts' own logits are at hand), greedy (share of sequences without sampling)
  keep     seqs, planes (layers x kv heads x 2), cap (rows of a plane), dim, tokens (of a tree)
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-6
BASE = 10000.0


def _rope(name=None, tokens=1, q_heads=32, kv_heads=8, dim=128, rot=128, pairs=False, norm=True, type="f16"):
    c = dict(op="rope", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=rot, pairs=pairs, norm=norm, type=type)
    return dict(c, name=name) if name else c


def _tree(name=None, seqs=1, tokens=16, branch=2, q_heads=32, kv_heads=8, dim=128, context=4096, ragged=False, type="f16"):
    c = dict(op="tree", seqs=seqs, tokens=tokens, branch=branch, q_heads=q_heads, kv_heads=kv_heads, dim=dim, context=context,
             ragged=ragged, type=type)
    return dict(c, name=name) if name else c


def _verify(name=None, seqs=1, tokens=5, branch=1, vocab=128256, drafts=True, greedy=0.0, type="f16"):
    c = dict(op="verify", seqs=seqs, tokens=tokens, branch=branch, vocab=vocab, drafts=drafts, greedy=greedy, type=type)
    return dict(c, name=name) if name else c


def _keep(name=None, seqs=1, planes=512, cap=4200, dim=128, tokens=16, type="f16"):
    c = dict(op="keep", seqs=seqs, planes=planes, cap=cap, dim=dim, tokens=tokens, type=type)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of the 8B-shaped stack's heads (launch latency)
        _rope("rope_1"),
        # a prompt chunk of the MoE stack's heads, half of each head rotated, neighbours paired, no norm
        _rope("rope_chunk_2047", 2047, 32, 4, 128, 64, True, False, "bf16"),
        # the largest prompt chunk of the tier table
        _rope("rope_prompt_16384", 16384),
        # the smallest tree, in the heads of the tests' miniature, over a short prompt (launch latency)
        _tree("tree_5_over_77", 1, 5, 2, 4, 2, 128, 77),
        # interactive decode, one sequence: a tree of 24 drafts over a 4K context
        _tree("tree_24_over_4096", 1, 24, 3),
        # a batch of sequences of several lengths with short chains of drafts, heads of 64
        _tree("tree_16_seqs_ragged", 16, 17, 1, 16, 8, 64, 8190, True, "bf16"),
        # a long document: a wide tree over 128K positions in the MoE stack's heads
        _tree("tree_64_over_131072", 1, 64, 4, 32, 4, 128, 131072),
        # a chain of four drafts of a small vocabulary, one sequence (launch latency)
        _verify("verify_chain_1", 1, 5, 1, 32000),
        # a batch of trees whose drafts are the draft model's best tokens; a part of the sequences does not sample
        _verify("verify_16_seqs_given", 16, 24, 3, 128256, False, 0.25, "bf16"),
        # a large batch of trees with the draft model's logits
        _verify("verify_32_seqs_drafts", 32, 32, 2, 128256, True),
        # one sequence of the 8B-shaped stack: 32 layers, 8 kv heads, K and V
        _keep("keep_1", 1, 512),
        # a batch that shares a cache
        _keep("keep_48_seqs", 48, 256, 301, 128, 24, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "tree", "tree", "verify", "verify", "keep"])
    kv = rng.choice([2, 4, 8])
    q = kv * rng.choice([1, 2, 4, 8]) if op == "tree" else kv * rng.choice([1, 3, 4, 8])
    if op == "rope":
        dim = rng.choice([64, 80, 128])
        rot = rng.choice([dim, dim // 2])
        return _rope(None, _log(rng, 1, 8191), q, kv, dim, rot, rng.random() < 0.3, rng.random() < 0.8, rng.choice(["f16", "bf16", "f32"]))
    if op == "tree":
        seqs = _log(rng, 1, 16)
        tokens = _log(rng, 1, 64)
        most = 131072 * 64 // (seqs * max(tokens, 16))
        return _tree(None, seqs, tokens, rng.choice([1, 2, 3]), min(q, 32), kv if min(q, 32) % kv == 0 else 4, rng.choice([64, 128]),
                     _log(rng, 40, max(41, min(65536, most))), rng.random() < 0.5, rng.choice(["f16", "bf16"]))
    if op == "verify":
        seqs = _log(rng, 1, 32)
        return _verify(None, seqs, _log(rng, 2, 32), rng.choice([1, 2, 3]), _log(rng, 1000, 131072), rng.random() < 0.5,
                       rng.choice([0.0, 0.0, 0.5]), rng.choice(["f16", "bf16", "f32"]) if seqs <= 8 else rng.choice(["f16", "bf16"]))
    seqs = _log(rng, 1, 48)
    return _keep(None, seqs, 2 * _log(rng, 8, 256), _log(rng, 100, 300), rng.choice([64, 128]), _log(rng, 2, 64), rng.choice(["f16", "bf16"]))


# ------------------------------------------------------------------ sizes that a case fixes

def _sizes(case):
    """Tokens of each sequence's tree: the largest, and where there are several sequences also smaller ones."""
    t, s = case["tokens"], case["seqs"]
    return [t - (5 * i) % max(1, (t + 1) // 2) for i in range(s)]


def _contexts(case):
    c, s = case["context"], case["seqs"]
    return [c if not case["ragged"] else max(0, c - (i * i * c) // (s * s)) for i in range(s)]


def _parents(t, branch):
    return [-1] + [(i - 1) // branch for i in range(1, t)]


def _inner(t, branch):
    return (t - 1 + branch - 1) // branch      # nodes that have children


def work(case):
    e = BYTES[case["type"]]
    if case["op"] == "rope":
        n = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        turned = 6 * case["rot"] // 2
        return {"bytes": 2.0 * n * case["dim"] * e, "flops": float(n * (turned + (4 * case["dim"] if case["norm"] else 0)))}
    if case["op"] == "tree":
        d, hq, hk = case["dim"], case["q_heads"], case["kv_heads"]
        ts, cs = _sizes(case), _contexts(case)
        rows = sum(2 * hk * c for c in cs) + sum(2 * hk * t + 2 * hq * t for t in ts)
        seen = sum(t * (c + 1) for t, c in zip(ts, cs))
        return {"bytes": float(rows * d * e), "flops": 4.0 * d * hq * seen}
    if case["op"] == "verify":
        # the rows of nodes with children, and of one last node of each sequence
        rows = sum(_inner(t, case["branch"]) for t in _sizes(case))
        rows = (2 if case["drafts"] else 1) * rows + case["seqs"]
        return {"bytes": float(rows * case["vocab"] * e), "flops": 10.0 * rows * case["vocab"]}
    moved = sum(len(p) - 1 for p in _paths(case))
    return {"bytes": 2.0 * moved * case["planes"] * case["dim"] * e, "flops": 0.0}


def _paths(case):
    """Accepted paths: node 0, then every second or third node."""
    return [list(range(0, t, 2 + i % 2))[:6] for i, t in enumerate(_sizes(case))]


# ------------------------------------------------------------------ inputs

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = dict(case=case)
    dt = TYPES[case["type"]]
    if case["op"] == "rope":
        n, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
        qkv = (_normal(g, n, (hq + 2 * hk) * d) * 2).to(dt)        # the rows that a QKV projection leaves
        s["q"], s["k"] = qkv[:, :hq * d].view(n, hq, d), qkv[:, hq * d:(hq + hk) * d].view(n, hk, d)
        start = torch.randint(0, 1 << 20, (1,), generator=g, device=DEVICE)
        s["positions"] = (start + torch.arange(n, device=DEVICE)).to(torch.int32)
        half = case["rot"] // 2
        s["inv_freq"] = torch.exp(torch.arange(half, device=DEVICE, dtype=torch.float64) * (-math.log(BASE) / half)).float()
        s["q_gain"] = (1 + 0.2 * _normal(g, d)).to(dt) if case["norm"] else None
        s["k_gain"] = (1 + 0.2 * _normal(g, d)).to(dt) if case["norm"] else None
        return s
    ts = _sizes(case)
    first = [sum(ts[:i]) for i in range(len(ts) + 1)]
    n, t_max = first[-1], max(ts)
    s["first"], s["t_max"] = _ints(first), t_max
    # where each row lies among its sequence's: for the plain forms, which work on padded sequences
    s["seq"] = torch.repeat_interleave(torch.arange(len(ts), device=DEVICE), torch.tensor(ts, device=DEVICE))
    s["slot"] = torch.arange(n, device=DEVICE) - s["first"][s["seq"]]
    if case["op"] == "keep":
        s["cache"] = _normal(g, case["seqs"], case["planes"], case["cap"], case["dim"]).to(dt)
        paths = _paths(case)
        s["path"] = _ints([p + [-1] * (t_max - len(p)) for p in paths])
        s["count"] = _ints([len(p) for p in paths])
        room = case["cap"] - t_max
        s["context"] = torch.randint(room // 2, room + 1, (case["seqs"],), generator=g, device=DEVICE).to(torch.int32)
        return s
    s["parent"] = _ints([p for t in ts for p in _parents(t, case["branch"])])
    if case["op"] == "tree":
        hq, hk, d, b = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]
        qkv = _normal(g, n, (hq + 2 * hk) * d).to(dt)
        s["q"] = (qkv[:, :hq * d] * 2).view(n, hq, d)
        s["k_new"], s["v_new"] = qkv[:, hq * d:(hq + hk) * d].view(n, hk, d), qkv[:, (hq + hk) * d:].view(n, hk, d)
        cap = case["context"] + t_max
        cache = torch.empty(b, hk, 2, cap, d, dtype=dt, device=DEVICE)      # K rows, then V rows, of every kv head
        for i in range(b):
            cache[i] = _normal(g, hk, 2, cap, d)
        s["k_cache"], s["v_cache"] = cache[:, :, 0], cache[:, :, 1]
        s["context"] = _ints(_contexts(case))
        return s
    v, b, br = case["vocab"], case["seqs"], case["branch"]
    s["temperature"] = torch.where(torch.arange(b, device=DEVICE) < round(case["greedy"] * b), 0.0, 0.8).float()
    target = torch.empty(n, v, dtype=dt, device=DEVICE)
    draft = torch.empty(n, v, dtype=dt, device=DEVICE)
    token = torch.zeros(n, dtype=torch.int32, device=DEVICE)
    for i in range(b):
        rows = slice(first[i], first[i + 1])
        x = _normal(g, ts[i], v) * 2.5
        target[rows] = x
        draft[rows] = 0.9 * x + 0.7 * _normal(g, ts[i], v)
        # the drafts: drawn from the parent's distribution, or its best tokens
        if ts[i] > 1:
            at = torch.tensor(_parents(ts[i], br)[1:], device=DEVICE)
            rank = (torch.arange(ts[i] - 1, device=DEVICE)) % br
            rows_p = draft[rows][at].float()
            if case["drafts"]:
                p = torch.softmax(rows_p / 0.8, -1)
                token[first[i] + 1:first[i + 1]] = torch.multinomial(p, 1, generator=g)[:, 0].int()
            else:
                token[first[i] + 1:first[i + 1]] = rows_p.topk(br, -1).indices.gather(1, rank[:, None])[:, 0].int()
    s["target"], s["token"] = target, token
    s["draft"] = draft if case["drafts"] else None
    s["u_accept"] = torch.rand(n, generator=g, device=DEVICE)
    s["u_sample"] = torch.rand(b, generator=g, device=DEVICE)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        from paper_2604_26334_amd import binding as B
        if case["op"] == "rope":
            return B.qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                                  eps=EPS, norm=case["norm"], pairs=case["pairs"])
        if case["op"] == "tree":
            return B.tree_attention(s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["first"], s["context"], s["parent"],
                                    max_context=case["context"], max_tree=s["t_max"])
        if case["op"] == "verify":
            return B.verify_tree(s["target"], s["token"], s["parent"], s["first"], s["u_accept"], s["u_sample"], draft_logits=s["draft"],
                                 temperature=s["temperature"], max_tree=s["t_max"], max_children=case["branch"])
        return B.cache_keep(s["cache"], s["path"], s["count"], s["context"])
    return {"rope": _plain_rope, "tree": _plain_tree, "verify": _plain_verify, "keep": _plain_keep}[case["op"]](s)


def _plain_rope(s):
    case = s["case"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()       # far positions: 64 bits
    return (_turned(s["q"], s["q_gain"], angle.cos().float(), angle.sin().float(), case),
            _turned(s["k"], s["k_gain"], angle.cos().float(), angle.sin().float(), case))


def _turned(x, gain, cos, sin, case):
    y = x.float()
    if case["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.float()
    r = case["rot"]
    if case["pairs"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., r:]), -1).to(x.dtype)


def _padded(x, s):
    """Rows [n, ...] -> [sequences, largest tree, ...]"""
    y = x.new_zeros(s["case"]["seqs"], s["t_max"], *x.shape[1:])
    y[s["seq"], s["slot"]] = x
    return y


def _ancestors(s):
    """[sequences, t, t]: whether a token is another one or comes behind it: the parents' table raised to a high power"""
    parent = torch.full((s["case"]["seqs"], s["t_max"]), -1, device=DEVICE, dtype=torch.int64)
    parent[s["seq"], s["slot"]] = s["parent"].long()
    eye = torch.eye(s["t_max"], device=DEVICE)
    near = eye + (parent[..., None] == torch.arange(s["t_max"], device=DEVICE)).float()
    for _ in range(max(1, math.ceil(math.log2(s["t_max"] + 1)))):
        near = (torch.matmul(near, near) > 0).float()
    return near > 0


def _plain_tree(s):
    case = s["case"]
    b, t, hq, hk, d = case["seqs"], s["t_max"], case["q_heads"], case["kv_heads"], case["dim"]
    c = case["context"]
    q = _padded(s["q"], s).float().view(b, t, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    kn, vn = (_padded(s[n], s).float().transpose(1, 2) for n in ("k_new", "v_new"))
    k = torch.cat((s["k_cache"][:, :, :c].float(), kn), 2)
    v = torch.cat((s["v_cache"][:, :, :c].float(), vn), 2)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    old = (torch.arange(c, device=DEVICE) < s["context"][:, None])[:, None, :].expand(b, t, c)
    seen = torch.cat((old, _ancestors(s)), 2)[:, None, None].expand(b, hk, hq // hk, t, c + t).reshape(b, hk, -1, c + t)
    scores.masked_fill_(~seen, -math.inf)
    scores -= scores.amax(-1, keepdim=True)
    w = scores.exp_()
    o = torch.matmul(w, v) / w.sum(-1, keepdim=True)
    o = o.view(b, hk, hq // hk, t, d).permute(0, 3, 1, 2, 4).reshape(b, t, hq, d)
    return o[s["seq"], s["slot"]].to(s["q"].dtype)


def _chances(logits, s):
    """Rows of probabilities in 64 bits (a border of their running sum lies among many); one token's alone where nothing is sampled"""
    temp = s["temperature"][s["seq"]][:, None].double()
    x = logits.double()
    best = torch.where(x == x.amax(-1, keepdim=True), torch.arange(x.shape[1], device=DEVICE), x.shape[1]).amin(-1)
    p = torch.softmax(x / torch.where(temp > 0, temp, 1.0), -1)
    return torch.where(temp > 0, p, (torch.arange(x.shape[1], device=DEVICE) == best[:, None]).double())


def _plain_verify(s):
    case = s["case"]
    n, b, t = s["seq"].numel(), case["seqs"], s["t_max"]
    row = torch.arange(n, device=DEVICE)
    token = s["token"].long()
    p = _chances(s["target"], s)
    q = _chances(s["draft"], s) if case["drafts"] else None
    up = s["parent"].long()
    at = torch.where(up >= 0, s["first"][s["seq"]].long() + up, n)        # the parent's row; node 0 has none
    # a node's children, in order: child[node, k]
    rank = torch.where(up >= 0, (s["slot"] - 1) % case["branch"], 0)
    child = torch.full((n + 1, case["branch"]), n, device=DEVICE)
    child[at, rank] = row
    child = child[:n]
    c, w = torch.zeros(n, device=DEVICE, dtype=torch.float64), torch.ones(n, device=DEVICE, dtype=torch.float64)
    went = torch.full((n,), n, device=DEVICE)                             # the accepted child's row
    rest = p.clone()                                                      # what is left to draw from, unscaled
    for k in range(case["branch"]):
        x = child[:, k]
        there = x < n
        tok = token[x.clamp(max=n - 1)]
        u = s["u_accept"][x.clamp(max=n - 1)].double()
        px = (p if case["drafts"] else rest).gather(1, tok[:, None])[:, 0]
        qx = q.gather(1, tok[:, None])[:, 0] if case["drafts"] else torch.ones_like(px)
        yes = there & (went == n) & (px > (c + u * w) * qx)
        went = torch.where(yes, x, went)
        no = there & (went == n)
        if case["drafts"]:
            # where nothing is sampled both rows are one token's: refused means that the two differ
            c = torch.where(no, c + w, c)
            left = (p - c[:, None] * q).clamp(min=0)
            sampled = (s["temperature"][s["seq"]] > 0)
            rest = torch.where((no & sampled)[:, None], left, rest)
            w = torch.where(no, torch.where(sampled, left.sum(-1), 1.0), w)
            c = torch.where(sampled, c, 0.0)
        else:
            sampled = (s["temperature"][s["seq"]] > 0)
            gone = torch.zeros_like(rest).scatter_(1, tok[:, None], 1.0).bool() & (no & sampled)[:, None]
            rest = rest.masked_fill(gone, 0)
            w = torch.where(no, rest.sum(-1), w)
    if case["drafts"]:      # without sampling the target's token alone decides
        greedy = ~(s["temperature"][s["seq"]] > 0)
        best = p.argmax(-1)
        hit = (token[child.clamp(max=n - 1)] == best[:, None]) & (child < n)
        first = torch.where(hit, child, n).amin(-1)
        went = torch.where(greedy, first, went)
    # the walk from node 0
    here = s["first"][:-1].long()
    path = torch.full((b, t), -1, device=DEVICE)
    path[:, 0] = 0
    for k in range(1, t):
        on = torch.cat((went, went.new_full((1,), n)))[here]
        on = torch.where(path[:, k - 1] < 0, n, on)
        path[:, k] = torch.where(on < n, on - s["first"][:-1], -1)
        here = torch.where(on < n, on, here)
    r = rest[here]
    run_sum = r.cumsum(-1)
    over = run_sum > s["u_sample"].double()[:, None] * run_sum[:, -1:]
    nxt = torch.where(over, torch.arange(r.shape[1], device=DEVICE), r.shape[1]).amin(-1)
    return path.int(), (path >= 0).sum(-1).int(), nxt.int()


def _plain_keep(s):
    cache, path = s["cache"], s["path"].long()
    b, t = path.shape
    i = torch.arange(t, device=DEVICE)
    ctx = s["context"].long()[:, None]
    live = i < s["count"][:, None]
    src = torch.where(live, ctx + path, ctx + i)
    at = torch.arange(b, device=DEVICE)[:, None]
    cache[at, :, ctx + i] = cache[at, :, src]
    return cache


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    if case["op"] == "verify":
        return None          # whole numbers
    s = prepare(case, seed)
    if case["op"] == "keep":
        out = s["cache"].double() if s["cache"].numel() < 1 << 26 else None
        if out is None:
            return None
        old = out.clone()
        for b, p in enumerate(_paths(case)):
            c = int(s["context"][b])
            for i, node in enumerate(p):
                out[b, :, c + i] = old[b, :, c + node]
        return out
    if case["op"] == "rope":
        got = []
        for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
            x = x.double()
            if case["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * gain.double()
            y = x.clone()
            for i in range(case["rot"] // 2):
                turn = s["positions"].double() * float(s["inv_freq"][i])
                co, si = torch.cos(turn)[:, None], torch.sin(turn)[:, None]
                a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + case["rot"] // 2)
                y[:, :, a] = x[:, :, a] * co - x[:, :, b] * si
                y[:, :, b] = x[:, :, a] * si + x[:, :, b] * co
            got.append(y)
        return tuple(got)
    if work(case)["flops"] > 4e12:
        return None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    group = case["q_heads"] // case["kv_heads"]
    first = s["first"].tolist()
    for b, (t, c) in enumerate(zip(_sizes(case), _contexts(case))):
        rows = slice(first[b], first[b + 1])
        parent = _parents(t, case["branch"])
        seen = torch.zeros(t, t, dtype=torch.bool)
        for i in range(t):
            j = i
            while j >= 0:
                seen[i, j] = True
                j = parent[j]
        seen = torch.cat((torch.ones(t, c, dtype=torch.bool), seen), 1).to(DEVICE)
        for h in range(case["kv_heads"]):
            k = torch.cat((s["k_cache"][b, h, :c], s["k_new"][rows, h])).double()
            v = torch.cat((s["v_cache"][b, h, :c], s["v_new"][rows, h])).double()
            for qh in range(h * group, (h + 1) * group):
                z = s["q"][rows, qh].double() @ k.T / math.sqrt(case["dim"])
                out[rows, qh] = torch.softmax(z.masked_fill(~seen, -math.inf), -1) @ v
    return out
