"""Operators of a step that answers several drafted tokens against the float64 oracle."""
import math

import numpy as np
import pytest

from oracle import drafts as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _t():
    import torch
    return torch


def _dt(name):
    torch = _t()
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


def _half_step(name):
    return _t().finfo(_dt(name)).eps / 2


def _np(t):
    return t.detach().double().cpu().numpy()


def _ints(v):
    torch = _t()
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _gen(seed):
    torch = _t()
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _same_bits(a, b):
    torch = _t()
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ------------------------------------------------------------------ norms and rotation

def _rope_tolerance(x, inv, pos, ref, norm, ty):
    """One rounding to the type (half a step of the value), and fp32 in front of it: the sum of squares of d terms (d / 2 steps of its half
    in the root), the root, its inverse and two products (2 steps each), sine and cosine of an angle exact to 2^-24 or so (4 steps
    allowed), two products and a sum; each of the pair's values takes part, so it goes by the pair's length.  24 + d steps in all."""
    d = x.shape[-1]
    half = len(inv)
    length = np.abs(ref)
    if half:
        size = np.abs(ref).max(-1, keepdims=True)
        length = np.broadcast_to(size, ref.shape)
    return np.abs(ref) * _half_step(ty) + length * 1.5 * (24 + d) * 2.0 ** -24 + 1e-7


@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,pairs,norm,gain,lay", [
    (1, 4, 2, 128, 128, False, True, True, "rows"), (1, 32, 8, 128, 128, False, True, True, "qkv"), (5, 3, 1, 64, 64, True, True, True, "qkv"),
    (7, 2, 2, 80, 40, False, True, False, "qkv"), (3, 4, 2, 80, 80, True, False, False, "rows"), (2, 1, 0, 96, 2, False, True, True, "rows"),
    (3, 0, 3, 256, 64, True, True, True, "rows"), (4, 2, 1, 7, 6, False, True, True, "odd"), (4, 2, 1, 128, 96, False, True, True, "odd"),
    (65, 5, 3, 128, 128, False, True, True, "odd"), (2, 2, 1, 512, 512, False, True, True, "rows"), (2, 2, 1, 1, 0, False, True, True, "rows"),
    (3, 2, 1, 128, 0, False, True, True, "rows"), (3, 2, 1, 64, 64, False, False, True, "heads"), (130, 8, 4, 64, 32, True, True, True, "heads"),
    (33, 24, 8, 128, 128, False, True, True, "in place"), (9, 3, 1, 128, 64, True, True, True, "in place")])
def test_rope(ty, tokens, hq, hk, d, rot, pairs, norm, gain, lay):
    from paper_2604_26334_amd import binding as B
    torch = _t()
    g = _gen(tokens * 1000 + d)
    dt = _dt(ty)

    def laid(heads):
        x = torch.randn(tokens, heads, d, generator=g, device=DEV) * 2
        if lay == "heads":        # heads first in memory
            return x.to(dt).transpose(0, 1).contiguous().transpose(0, 1)
        if lay == "odd":          # rows that start anywhere
            buf = torch.zeros(tokens * heads * (d + 1) + 1, dtype=dt, device=DEV)
            y = buf[1:].view(tokens, heads, d + 1)[:, :, :d]
            y.copy_(x)
            return y
        return x.to(dt)
    q, k = laid(hq), laid(hk)
    if lay == "qkv":              # as a projection leaves them
        row = torch.cat((q.reshape(tokens, -1), k.reshape(tokens, -1), k.reshape(tokens, -1)), 1).contiguous()
        q, k = row[:, :hq * d].view(tokens, hq, d), row[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
    pos = torch.tensor([(i * 7919 + 1) % 1000003 if i % 3 else -i for i in range(tokens)], dtype=torch.int32, device=DEV)
    inv = torch.tensor(np.exp(-np.arange(rot // 2) / max(1, rot // 2) * math.log(10000.0)), dtype=torch.float32, device=DEV)
    gq = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt) if gain else None
    gk = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt) if gain else None
    xq, xk = _np(q), _np(k)
    out = dict(q_out=q, k_out=k) if lay == "in place" else {}
    a, b = B.qk_norm_rope(q, k, pos if rot else None, inv if rot else None, q_gain=gq, k_gain=gk, norm=norm, pairs=pairs, **out)
    torch.cuda.synchronize()
    if lay == "in place":
        assert a.data_ptr() == q.data_ptr() and b.data_ptr() == k.data_ptr()
    for got, x, gn in ((a, xq, gq), (b, xk, gk)):
        if got.numel() == 0:
            continue
        ref = D.qk_norm_rope(x, None if gn is None else _np(gn), pos.tolist(), inv.cpu().numpy(), 1e-6, norm, pairs)
        off = np.abs(_np(got) - ref) / _rope_tolerance(x, inv.cpu().numpy(), pos, ref, norm, ty)
        assert off.max() <= 1, off.max()


def test_rope_of_zero_rows_infinities_and_neighbours():
    """A row of zeros stays zero; an infinite or missing number stays in its own head; memory between and behind rows stays."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for d, step in ((128, 256), (128, 131), (66, 67)):
        buf = torch.full((4, 3, step), 7.0, dtype=torch.float16, device=DEV)
        x = buf[:, :, :d]
        x.copy_(torch.randn(4, 3, d, generator=_gen(1), device=DEV))
        x[0, 0] = 0
        x[1, 1, 5] = float("inf")
        x[2, 2, 6] = float("nan")
        ref = D.qk_norm_rope(_np(x[3]).reshape(1, 3, d), None, [12], np.float32([1.0] * (d // 2)), 1e-6, True, False)
        pos = torch.tensor([3, 4, 5, 12], dtype=torch.int32, device=DEV)
        got, _ = B.qk_norm_rope(x, x[:, :0], pos, torch.ones(d // 2, device=DEV), q_out=x, k_out=x[:, :0])
        torch.cuda.synchronize()
        assert bool((buf[:, :, d:] == 7).all())
        assert bool((got[0, 0] == 0).all()) and np.abs(_np(got[3:]) - ref).max() < 5e-3
        fine = torch.isfinite(got).all(-1).cpu().numpy()
        want = np.ones((4, 3), bool)
        want[1, 1] = want[2, 2] = False
        assert (fine == want).all()


# ------------------------------------------------------------------ tree attention

def _random_parents(rng, t, kind):
    if kind == "chain":
        return [i - 1 for i in range(t)]
    if kind == "flat":
        return [-1] * t
    if kind == "wild":           # values that no tree has count as none
        return [int(rng.choice([i, i + 1, -7, 2 ** 31 - 1, -2 ** 31])) if rng.random() < 0.3 else int(rng.integers(-1, max(1, i))) for i in range(t)]
    return [-1][:t] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, t)]


def _attention_case(ty, d, hq, hk, trees, ctxs, cap, kind="tree", seed=0, sharp=1.0, lay="qkv", pad=0):
    torch = _t()
    g, rng, dt = _gen(seed + 17), np.random.default_rng(seed), _dt(ty)
    n = sum(trees) + pad
    qkv = torch.randn(n, (hq + 2 * hk) * d, generator=g, device=DEV)
    qkv[:, :hq * d] *= sharp
    qkv = qkv.to(dt)
    q, kn, vn = (qkv[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    b = len(trees)
    if lay == "rows":            # positions first: [sequence][position][head]
        kc = torch.randn(b, cap, hk, d, generator=g, device=DEV).to(dt).transpose(1, 2)
        vc = torch.randn(b, cap, hk, d, generator=g, device=DEV).to(dt).transpose(1, 2)
    else:                        # the stack's: K rows then V rows of every kv head
        cache = torch.randn(b, hk, 2, cap, d, generator=g, device=DEV).to(dt)
        kc, vc = cache[:, :, 0], cache[:, :, 1]
    for i, c in enumerate(ctxs):        # what lies behind the context is never read
        kc[i, :, c:] = float("nan")
        vc[i, :, c:] = float("inf")
    first = np.concatenate([[0], np.cumsum(trees)]).tolist()
    parent = [p for t in trees for p in _random_parents(rng, t, kind)] + [0] * pad
    return dict(q=q, k_new=kn, v_new=vn, k_cache=kc, v_cache=vc, first=_ints(first), context=_ints(ctxs), parent=_ints(parent)), first, parent


def _attention_tolerance(ref, v_max, scores, ty):
    """Half a step of the result; the weights' roundings (half a step of the type each, against a sum of the rounded ones: their errors move the
    result by at most half a step of the spread of the values, 2 v_max); and scores in fp32: head_dim terms, their sum's error
    and that of the exponential's argument are at most (head_dim + 8) 2^-24 of the terms' size, which moves weights by that much."""
    return np.abs(ref) * _half_step(ty) + 2 * v_max * (_half_step(ty) + scores * 2.0 ** -24)


def _check_attention(a, out, first, parent, trees, ctxs, ty, d, scale):
    for s, (t, c) in enumerate(zip(trees, ctxs)):
        if t == 0:
            continue
        r = slice(first[s], first[s] + t)
        q, kn, vn, kc, vc = _np(a["q"][r]), _np(a["k_new"][r]), _np(a["v_new"][r]), _np(a["k_cache"][s, :, :c]), _np(a["v_cache"][s, :, :c])
        ref = D.tree_attention(q, kn, vn, kc, vc, c, parent[r], scale)
        v_max = max(np.abs(vn).max(), np.abs(vc).max() if c else 0)
        k_max = max(np.abs(kn).max(), np.abs(kc).max() if c else 0)
        size = np.abs(q).sum(-1).max() * k_max * abs(scale) * 4
        tol = _attention_tolerance(ref, v_max, size * (d + 8) / d + 8, ty)
        off = np.abs(_np(out[r]) - ref) / tol
        assert off.max() <= 1, (s, t, c, off.max())


TREES = [
    # d, q heads, kv heads, trees, contexts, capacity, kind
    (128, 4, 2, [1], [0], 4, "chain"), (128, 4, 2, [1], [1], 4, "chain"), (128, 32, 8, [1], [257], 300, "chain"),
    (128, 4, 2, [5], [77], 100, "tree"), (64, 4, 4, [5], [31], 40, "tree"), (128, 8, 1, [3, 0, 2], [32, 10, 33], 64, "tree"),
    (128, 4, 1, [16, 1, 7], [0, 128, 129], 160, "tree"), (64, 16, 8, [17, 12, 17], [500, 3, 127], 520, "chain"),
    (128, 6, 2, [33], [200], 240, "tree"), (128, 32, 4, [24], [1030], 1060, "tree"), (64, 12, 1, [64], [64], 128, "flat"),
    (128, 4, 4, [64, 63], [96, 95], 160, "wild"), (128, 8, 2, [256], [40], 300, "chain"), (64, 2, 2, [200, 256], [0, 70], 330, "tree"),
    (128, 3, 1, [9] * 20, [i * 13 % 90 for i in range(20)], 110, "tree"), (128, 64, 1, [20], [300], 330, "tree"),
    (64, 1, 1, [255], [511], 768, "wild"),
]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("case", range(len(TREES)))
def test_tree_attention(ty, case):
    from paper_2604_26334_amd import binding as B
    d, hq, hk, trees, ctxs, cap, kind = TREES[case]
    a, first, parent = _attention_case(ty, d, hq, hk, trees, ctxs, cap, kind, case, sharp=(1.0, 4.0)[case % 2], lay=("qkv", "rows")[case // 2 % 2])
    out = B.tree_attention(**a, max_context=max(ctxs), max_tree=max(trees))
    _check_attention(a, out, first, parent, trees, ctxs, ty, d, d ** -0.5)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("d,hq,hk,t,ctx", [(128, 32, 8, 1, 4097), (128, 8, 2, 24, 9000), (64, 16, 2, 64, 5003), (128, 16, 4, 7, 70001)])
def test_tree_attention_over_long_contexts(ty, d, hq, hk, t, ctx):
    """Sharp scores, so that single positions weigh; the boundaries' positions are each some row's favourite."""
    from paper_2604_26334_amd import binding as B
    a, first, parent = _attention_case(ty, d, hq, hk, [t], [ctx], ctx + t, "tree", ctx, sharp=3.0)
    spots = [0, 31, 32, 127, 128, 4095, ctx // 2, ctx - 33, ctx - 32, ctx - 1]
    for i, p in enumerate(spots):
        p = min(max(p, 0), ctx - 1)
        a["k_cache"][0, :, p] = a["q"][i % t, ::hq // hk] * 0.7
    out = B.tree_attention(**a, max_context=ctx, max_tree=t)
    _check_attention(a, out, first, parent, [t], [ctx], ty, d, d ** -0.5)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_hidden_tokens_may_hold_anything(ty):
    """A node that is no ancestor does not count, whatever its key and value hold; one that is does."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for bad in (float("nan"), float("inf"), torch.finfo(_dt(ty)).min):
        a, first, _ = _attention_case(ty, 128, 4, 2, [6], [37], 64, "chain", 3)
        parent = [-1, 0, 0, 1, 2, 3]                    # two branches: 0 1 3 5 and 0 2 4
        a["parent"] = _ints(parent)
        clean = B.tree_attention(**a, max_context=40, max_tree=6)
        for key in (True, False):
            k, v = a["k_new"].clone(), a["v_new"].clone()
            if key:
                k[2] = bad
            v[2] = bad
            out = B.tree_attention(**dict(a, k_new=k, v_new=v), max_context=40, max_tree=6)
            assert _same_bits(out[[0, 1, 3, 5]], clean[[0, 1, 3, 5]]), (bad, key)
            if not math.isfinite(bad) and not key:
                assert not bool(torch.isfinite(out[[2, 4]]).any()), bad


@pytest.mark.parametrize("t,hq", [(3, 2), (24, 4), (9, 16)])
def test_keys_that_are_no_numbers_reach_every_row_that_sees_them(t, hq):
    """A run of cached keys without a number, as long as a whole tile, step or split: no row may come out finite."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for lo, hi in ((0, 32), (32, 64), (64, 192), (0, 700), (640, 700)):
        a, first, _ = _attention_case("f16", 128, hq, 2, [t], [700], 740, "tree", 3)
        a["k_cache"][0, 1, lo:hi] = float("nan")
        out = B.tree_attention(**a, max_context=700, max_tree=t)
        fine = torch.isfinite(out).all(-1)
        assert bool(fine[:, :hq // 2].all()) and not bool(fine[:, hq // 2:].any()), (lo, hi)


@pytest.mark.parametrize("t,hq", [(3, 2), (24, 4)])
@pytest.mark.parametrize("scale", [-0.09, 0.0, 1.3])
def test_tree_attention_with_any_scale(t, hq, scale):
    from paper_2604_26334_amd import binding as B
    a, first, parent = _attention_case("bf16", 128, hq, 2, [t, t], [333, 40], 400, "tree", 6)
    out = B.tree_attention(**a, max_context=333, max_tree=t, scale=scale)
    _check_attention(a, out, first, parent, [t, t], [333, 40], "bf16", 128, scale)


def test_tree_attention_of_padded_batches_and_bounded_values():
    """Rows behind the last sequence keep what they hold; contexts, offsets and lengths out of range are bounded as documented."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    a, first, parent = _attention_case("f16", 128, 4, 2, [5, 0, 4], [20, 3, 30], 64, "tree", 5, pad=7)
    out = torch.full((16, 4, 128), 3.0, dtype=torch.float16, device=DEV)
    B.tree_attention(**a, max_context=30, max_tree=5, out=out)
    _check_attention(a, out, first, parent, [5, 0, 4], [20, 3, 30], "f16", 128, 128 ** -0.5)
    assert bool((out[9:] == 3).all())
    # longer contexts count as max_context, negative ones as none; tokens beyond max_tree are left out
    out.fill_(3.0)
    B.tree_attention(**dict(a, context=_ints([2 ** 31 - 1, 0, -5])), max_context=19, max_tree=4, out=out)
    _check_attention(a, out, first, parent, [4, 0, 4], [19, 0, 0], "f16", 128, 128 ** -0.5)
    assert bool((out[4] == 3).all()) and bool((out[9:] == 3).all())
    # offsets: bounded to the tokens there are; a sequence that ends before it starts has none
    out.fill_(3.0)
    B.tree_attention(**dict(a, first=_ints([12, 2 ** 31 - 1, 7, -3])), max_context=30, max_tree=6, out=out)
    assert bool((out[:12] == 3).all()) and bool(torch.isfinite(out).all()) and not bool((out[12:] == 3).all())


@pytest.mark.parametrize("ty,d,hq,hk", [("f16", 128, 8, 2), ("bf16", 64, 4, 4)])
def test_tree_attention_appends_its_rows(ty, d, hq, hk):
    from paper_2604_26334_amd import binding as B
    torch = _t()
    trees, ctxs, cap = [5, 0, 70, 1], [20, 3, 300, 0], 400
    a, first, parent = _attention_case(ty, d, hq, hk, trees, ctxs, cap, "tree", 9)
    before_k, before_v = a["k_cache"].clone(), a["v_cache"].clone()
    plain = B.tree_attention(**a, max_context=300, max_tree=70)
    assert _same_bits(before_k, a["k_cache"].contiguous()) and _same_bits(before_v, a["v_cache"].contiguous())
    out = B.tree_attention(**a, max_context=300, max_tree=70, append=True)
    assert _same_bits(plain, out)
    for s, (t, c) in enumerate(zip(trees, ctxs)):
        r = slice(first[s], first[s] + t)
        before_k[s, :, c:c + t] = a["k_new"][r].transpose(0, 1)
        before_v[s, :, c:c + t] = a["v_new"][r].transpose(0, 1)
    assert _same_bits(before_k, a["k_cache"].contiguous()) and _same_bits(before_v, a["v_cache"].contiguous())


def test_tree_attention_does_not_depend_on_its_neighbours():
    """A sequence's rows are the same bits whatever else is in the batch, and in every run."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    a, first, _ = _attention_case("f16", 128, 8, 2, [9, 9, 9], [1000, 40, 700], 1100, "tree", 11)
    out = B.tree_attention(**a, max_context=1000, max_tree=9)
    assert _same_bits(out, B.tree_attention(**a, max_context=1000, max_tree=9))
    perm = [2, 0, 1]
    rows = torch.cat([torch.arange(first[p], first[p] + 9) for p in perm]).to(DEV)
    b = {n: a[n][rows].contiguous() for n in ("q", "k_new", "v_new", "parent")}
    b.update({n: a[n][perm].contiguous() for n in ("k_cache", "v_cache", "context")})
    assert _same_bits(out[rows], B.tree_attention(**b, first=a["first"], max_context=1000, max_tree=9))


def test_tree_attention_far_into_a_large_cache():
    """Offsets past 32 bits: positions first, so a row is 512 KB behind the one before it."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    hk, d, cap = 2048, 128, 9000               # 4.7 GB of K
    kc = torch.zeros(1, cap, hk, d, dtype=torch.float16, device=DEV).transpose(1, 2)
    t, ctx, g = 3, 8990, _gen(4)
    heads = slice(2046, 2048)
    sub = torch.randn(1, 2, cap, d, generator=g, device=DEV).half()
    kc[:, heads] = sub
    q = torch.randn(t, 2, d, generator=g, device=DEV).half() * 3
    kn, vn = (torch.randn(t, 2, d, generator=g, device=DEV).half() for _ in range(2))
    a = dict(q=q, k_new=kn, v_new=vn, k_cache=kc[:, heads], v_cache=kc[:, heads], first=_ints([0, t]), context=_ints([ctx]), parent=_ints([-1, 0, 0]))
    out = B.tree_attention(**a, max_context=ctx, max_tree=t)
    _check_attention(a, out, [0, t], [-1, 0, 0], [t], [ctx], "f16", d, d ** -0.5)


# ------------------------------------------------------------------ verification

def _verify_case(ty, rng, trees, V, kind="tree", drafts=True, temps=None, odd=False, spread=2.0, pad=0):
    torch = _t()
    n, dt = sum(trees) + pad, _dt(ty)
    target = torch.tensor(rng.normal(size=(n, V)) * spread, device=DEV).to(dt)
    draft = (target.double() * 0.9 + torch.tensor(rng.normal(size=(n, V)) * 0.5, device=DEV)).to(dt)
    if odd:              # rows that start anywhere
        wide = torch.zeros(n, V + 3, dtype=dt, device=DEV)
        wide[:, 1:V + 1] = target
        target = wide[:, 1:V + 1]
    first = np.concatenate([[0], np.cumsum(trees)]).tolist()
    parent = [p for t in trees for p in _random_parents(rng, t, kind)] + [0] * pad
    temp = [1.0] * len(trees) if temps is None else temps
    token = []
    dn = _np(draft)
    for s, t in enumerate(trees):
        for i in range(t):
            up = parent[first[s] + i]
            if 0 <= up < i:
                row = D._row(dn[first[s] + up], temp[s] if temp[s] > 0 else 0.5)
                token.append(int(rng.choice(V, p=row)) if drafts else int(np.argsort(-row, kind="stable")[rng.integers(0, min(V, 3))]))
            else:
                token.append(int(rng.integers(0, V)))
    token += [0] * pad
    return dict(target_logits=target, draft_logits=draft if drafts else None, token=_ints(token), parent=_ints(parent), first=_ints(first),
                u_accept=torch.tensor(rng.random(n), dtype=torch.float32, device=DEV),
                u_sample=torch.tensor(rng.random(len(trees)), dtype=torch.float32, device=DEV),
                temperature=None if temps is None else torch.tensor(temps, dtype=torch.float32, device=DEV)), first


def _check_verify(a, got, first, trees, max_tree, max_children=256):
    path, count, nxt = (t.cpu().tolist() for t in got)
    target, draft = _np(a["target_logits"]), None if a["draft_logits"] is None else _np(a["draft_logits"])
    token, parent = a["token"].tolist(), a["parent"].tolist()
    ua, us = a["u_accept"].tolist(), a["u_sample"].tolist()
    lengths = []
    for s, t in enumerate(trees):
        t = min(t, max_tree)
        r = slice(first[s], first[s] + t)
        temp = 1.0 if a["temperature"] is None else float(a["temperature"][s])
        want, n = D.verify_tree(target[r], token[r], parent[r], ua[r], us[s], None if draft is None else draft[r], temp, max_children)
        assert path[s] == want + [-1] * (max_tree - len(want)) and count[s] == len(want) and nxt[s] == n, (s, path[s], want, nxt[s], n)
        lengths.append(len(want))
    return lengths


@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("trees,V,kind,odd", [
    ([1], 1, "chain", False), ([2, 1, 0, 4], 2, "tree", False), ([5, 3], 33, "chain", True), ([12] * 6, 1000, "tree", False), ([7, 0, 9, 1], 4097, "tree", True),
    ([24, 24, 11], 32003, "tree", False), ([64, 3], 513, "wild", True), ([256, 100], 65, "flat", False), ([5] * 40, 257, "chain", False)])
def test_verify(ty, drafts, trees, V, kind, odd):
    from paper_2604_26334_amd import binding as B
    rng = np.random.default_rng(V * 10 + len(trees) + drafts)
    temps = [(1.0, 0.7, 0.0, 1.9, float("nan"))[i % 5] for i in range(len(trees))]
    a, first = _verify_case(ty, rng, trees, V, kind, drafts, [t if t == t else 0.0 for t in temps], odd, pad=3)
    got = B.verify_tree(**a, max_tree=max(trees))
    _check_verify(a, got, first, trees, max(trees))
    # the same with bounds that hide a part of the tree
    few = max(1, max(trees) - 2)
    got = B.verify_tree(**a, max_tree=few, max_children=2)
    _check_verify(a, got, first, trees, few, 2)


@pytest.mark.parametrize("drafts", [True, False])
def test_verify_a_large_vocabulary(drafts):
    from paper_2604_26334_amd import binding as B
    rng = np.random.default_rng(5)
    for V, spread in ((128256, 2.5), (151936, 0.01)):
        a, first = _verify_case("f16", rng, [9, 4, 1], V, "tree", drafts, [0.8, 1.0, 1.3], spread=spread)
        _check_verify(a, B.verify_tree(**a, max_tree=9, max_children=4), first, [9, 4, 1], 9, 4)


def test_verify_draws_at_the_borders():
    """Random numbers at both ends; every index of a small vocabulary is drawn where its share of the running sum lies."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    V, n = 300, 600
    u = np.float32([0, 1 - 2.0 ** -24, 2.0 ** -24] + list((np.arange(n - 3) + 0.5) / (n - 3)))
    row = np.random.default_rng(1).normal(size=V) * 2
    row[:3] = -np.inf
    row[-4:] = -np.inf
    a = dict(target_logits=torch.tensor(row, device=DEV).float().expand(n, V), draft_logits=None, token=_ints([0] * n), parent=_ints([-1] * n),
             first=_ints(list(range(n + 1))), u_accept=torch.zeros(n, device=DEV), u_sample=torch.tensor(u, device=DEV), temperature=None)
    got = B.verify_tree(**a, max_tree=1)
    _check_verify(a, got, list(range(n)), [1] * n, 1)
    assert got[2][0] == 3 and got[2][1] == V - 5


def test_verify_infinities_and_masks():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    inf, nan = float("inf"), float("nan")
    V = 70
    rng = np.random.default_rng(3)
    for ty in ("f16", "bf16", "f32"):
        for drafts in (True, False):
            a, first = _verify_case(ty, rng, [4] * 12, V, "tree", drafts, [1.0, 0.0] * 6)
            t = a["target_logits"]
            low = torch.finfo(_dt(ty)).min
            t[0:8] = -inf                       # nothing left
            t[8:16] = low                       # the lowest value everywhere: all alike
            t[16:24, 5:] = low                  # but for five
            t[24:32, ::2] = nan
            t[32:40, 3] = inf
            t[32:40, 9] = inf
            t[40:48] = -inf
            t[40:48, V - 1] = 0.5               # one left
            if drafts:
                a["draft_logits"][16:48] = -inf
                a["draft_logits"][16:20, 7] = 1
                a["draft_logits"][8:12] = nan
            got = B.verify_tree(**a, max_tree=4)
            _check_verify(a, got, first, [4] * 12, 4)
            assert got[2][0] == -1 and got[1][0] == 1 and got[2][11] == V - 1


def test_verify_tokens_out_of_range_and_twice():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    rng = np.random.default_rng(8)
    for drafts in (True, False):
        a, first = _verify_case("f32", rng, [8] * 30, 6, "flat", drafts)
        a["parent"] = _ints([-1, 0, 0, 0, 0, 0, 0, 0] * 30)
        a["token"] = _ints([int(x) for x in rng.choice([-1, 0, 1, 2, 2, 5, 6, 2 ** 31 - 1, -2 ** 31], size=240)])
        _check_verify(a, B.verify_tree(**a, max_tree=8), first, [8] * 30, 8)


def test_verify_bounds_its_offsets():
    from paper_2604_26334_amd import binding as B
    rng = np.random.default_rng(9)
    a, _ = _verify_case("f16", rng, [6, 6], 50, "tree", True)
    a["first"] = _ints([9, 2 ** 31 - 1, -4])
    path, count, nxt = B.verify_tree(**a, max_tree=6)
    assert path[0][0] == 0 and 1 <= int(count[0]) <= 3 and 0 <= int(nxt[0]) < 50
    assert path[1].tolist() == [-1] * 6 and int(count[1]) == 0 and int(nxt[1]) == -1


# ------------------------------------------------------------------ kept rows

@pytest.mark.parametrize("ty,planes,cap,d,width", [("f16", 3, 40, 64, 8), ("bf16", 5, 600, 128, 256), ("f32", 1, 20, 4, 3), ("f16", 9, 300, 2048, 64),
                                                   ("bf16", 130, 64, 128, 16)])
def test_keep(ty, planes, cap, d, width):
    from paper_2604_26334_amd import binding as B
    torch = _t()
    rng = np.random.default_rng(planes)
    seqs = 6
    cache = torch.randn(seqs, planes, cap, d, generator=_gen(2), device=DEV).to(_dt(ty))
    paths = [sorted(rng.choice(width, size=min(width, 5), replace=False).tolist()), list(range(width)), [], [0] * min(3, width),
             rng.integers(0, width, size=width).tolist(), list(range(width))[::-1]]
    ctx = [0, cap - width, 3, 1, (cap - width) // 2, max(0, cap - width)]
    want = cache.clone()
    for s, p in enumerate(paths):
        for i, node in enumerate(p):
            want[s, :, ctx[s] + i] = cache[s, :, ctx[s] + node]
    path = _ints([p + [-1] * (width - len(p)) for p in paths])
    B.cache_keep(cache, path, _ints([len(p) for p in paths]), _ints(ctx))
    assert _same_bits(cache, want)


def test_keep_leaves_out_what_lies_outside():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    wide = torch.randn(2, 3, 10, 24, generator=_gen(3), device=DEV).half()
    cache = wide[:, :, :, 8:16]                       # rows of 16 bytes inside longer ones
    want = wide.clone()
    w = want[:, :, :, 8:16]
    for i, node in ((1, 3), (3, 2)):                  # entries -1 and 9 are left out; row 6 + 4 lies outside
        w[0, :, 6 + i] = cache[0, :, 6 + node]
    B.cache_keep(cache, _ints([[-1, 3, 9, 2, 1], [2, 1, 0, 0, 0]]), _ints([5, 2 ** 31 - 1]), _ints([6, -4]))
    # sequence 1: rows -4 .. 0 of which only entries with both rows inside count: none (row -4 + 4 = 0 takes row -4)
    assert _same_bits(wide, want)
    before = wide.clone()
    B.cache_keep(cache, _ints([[1, 2, 3, 4, 0]] * 2), _ints([-3, 0]), _ints([2, 2]))
    assert _same_bits(wide, before)


# ------------------------------------------------------------------ together, on streams and in graphs

def _step(a, B, cache_planes):
    """rotation -> attention (appending) -> verification -> kept rows, as a serving loop calls them"""
    q, k = B.qk_norm_rope(a["q0"], a["k0"], a["positions"], a["inv_freq"], q_gain=a["gain"], k_gain=a["gain"])
    out = B.tree_attention(q, k, a["v"], a["k_cache"], a["v_cache"], a["first"], a["context"], a["parent"], max_context=200, max_tree=12, append=True)
    logits = (out.reshape(out.shape[0], -1).float() @ a["head"]).half()
    path, count, nxt = B.verify_tree(logits, a["token"], a["parent"], a["first"], a["u"], a["us"], draft_logits=a["draft"], max_tree=12, max_children=3)
    B.cache_keep(cache_planes, path, count, a["context"])
    return out, logits, path, count, nxt


def _step_case(seed):
    torch = _t()
    g, rng = _gen(seed), np.random.default_rng(seed)
    trees, n, hq, hk, d, V = [12, 5, 9], 26, 4, 2, 64, 777
    parent = [p for t in trees for p in _random_parents(rng, t, "tree")]
    cache = torch.randn(3, 2 * hk, 230, d, generator=g, device=DEV).half()
    f = lambda *s: torch.randn(*s, generator=g, device=DEV)      # noqa: E731
    return dict(q0=f(n, hq, d).half(), k0=f(n, hk, d).half(), v=f(n, hk, d).half(), gain=(1 + 0.1 * f(d)).half(),
                positions=_ints(list(range(190, 190 + n))), inv_freq=torch.exp(-torch.arange(d // 2, device=DEV) / 5.0), cache=cache,
                k_cache=cache[:, 0::2], v_cache=cache[:, 1::2], first=_ints([0, 12, 17, 26]), context=_ints([200, 3, 117]), parent=_ints(parent),
                head=f(hq * d, V) * 0.2, token=_ints(rng.integers(0, V, size=n).tolist()), u=torch.rand(n, generator=g, device=DEV) * 0.2,
                us=torch.rand(3, generator=g, device=DEV), draft=(f(n, V)).half())


def test_a_step_of_all_four():
    from paper_2604_26334_amd import binding as B
    a = _step_case(1)
    cache0 = a["cache"].clone()
    out, logits, path, count, nxt = _step(a, B, a["cache"])
    q = D.qk_norm_rope(_np(a["q0"]), _np(a["gain"]), a["positions"].tolist(), a["inv_freq"].cpu().numpy(), 1e-6, True, False)
    k = D.qk_norm_rope(_np(a["k0"]), _np(a["gain"]), a["positions"].tolist(), a["inv_freq"].cpu().numpy(), 1e-6, True, False)
    first, parent = a["first"].tolist(), a["parent"].tolist()
    for s, c in enumerate(a["context"].tolist()):
        r = slice(first[s], first[s + 1])
        ref = D.tree_attention(q[r], k[r], _np(a["v"][r]), _np(cache0[s, 0::2]), _np(cache0[s, 1::2]), c, parent[r], 64 ** -0.5)
        # queries and keys are rounded to fp16 in between (2^-11 each, scores of up to about 20: 0.02 of a weight)
        assert np.abs(_np(out[r]) - ref).max() < 0.02 * np.abs(ref).max() * 4
        want, n = D.verify_tree(_np(logits[r]), a["token"][r].tolist(), parent[r], a["u"][r].tolist(), float(a["us"][s]), _np(a["draft"][r]), 1.0)
        assert path[s].tolist()[:len(want)] == want and int(count[s]) == len(want) and int(nxt[s]) == n
        kept = _np(a["cache"][s, :, c:c + len(want)])
        kk, vv = k[r][want], _np(a["v"][r])[want]
        assert np.abs(kept[0::2] - kk.transpose(1, 0, 2)).max() <= np.abs(kk).max() * 2.0 ** -10
        assert np.array_equal(kept[1::2], vv.transpose(1, 0, 2))
        assert np.array_equal(_np(a["cache"][s, :, :c]), _np(cache0[s, :, :c]))


def test_a_step_on_another_stream_and_replayed():
    """The four as one captured graph, on a stream of its own: every replay gives the eager call's bits, with eager calls and other inputs in between."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    a = _step_case(2)
    start = a["cache"].clone()
    want = [t.clone() for t in _step(a, B, a["cache"])] + [a["cache"].clone()]
    other = _step_case(3)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a["cache"].copy_(start)
        got = _step(a, B, a["cache"])
        stream.synchronize()
        for x, y in zip(list(got) + [a["cache"]], want):
            assert _same_bits(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = _step(a, B, a["cache"])
    for i in range(4):
        a["cache"].copy_(start)
        for t in res:
            t.zero_()
        _step(other, B, other["cache"])
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(list(res) + [a["cache"]], want):
            assert _same_bits(x, y), i
    # new inputs in the same places
    for name in ("q0", "k0", "v", "u", "draft", "parent", "token", "context"):
        a[name].copy_(other[name])
    a["cache"].copy_(start)
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in res] + [a["cache"].clone()]
    a["cache"].copy_(start)
    for x, y in zip(list(_step(a, B, a["cache"])) + [a["cache"]], replayed):
        assert _same_bits(x, y)
