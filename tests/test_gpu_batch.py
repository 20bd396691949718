"""Operators of a step that answers a batch of requests over one paged cache against the float64 oracle."""
import numpy as np
import pytest

from oracle import batch as O
from tests.test_gpu_drafts import DEV, _attention_tolerance, _dt, _gen, _ints, _np, _same_bits, _t

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ places of new tokens

def _tables_case(seed, seqs, most_new, most_cached, page, n_pages=None, free=None, width=None, wild=False):
    rng = np.random.default_rng(seed)
    cached = [int(rng.integers(0, most_cached + 1)) if rng.random() < 0.8 else 0 for _ in range(seqs)]
    new = [int(rng.integers(0, most_new + 1)) for _ in range(seqs)]
    held = [-(-c // page) for c in cached]
    full = [-(-(c + n) // page) for c, n in zip(cached, new)]
    need = sum(full) - sum(held)
    n_pages = sum(full) + 5 if n_pages is None else n_pages
    order = [int(x) for x in rng.permutation(max(n_pages, sum(full) + 5))]
    width = max(full) + 1 if width is None else width
    table, at = [], 0
    for h in held:
        table.append([order[at + i] if i < h else int(rng.integers(-5, 5)) for i in range(width)])
        at += h
    free_pages = order[at:at + need + 5] if free is None else order[at:at + free]
    if wild:
        free_pages = [int(rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31])) if rng.random() < 0.3 else p for p in free_pages]
    return cached, new, table, free_pages, n_pages


def _run_tables(B, cached, new, table, free_pages, free_at, page, n_pages, n_tokens, offset=None, strided=False):
    torch = _t()
    width = len(table[0])
    if strided:
        buf = torch.full((len(table), width + 3), 77, dtype=torch.int32, device=DEV)
        t = buf[:, :width]
        t.copy_(_ints(table))
    else:
        t = _ints(table)
    out = {n: torch.full((m,), -9, dtype=torch.int32, device=DEV) for n, m in (("first", len(cached) + 1), ("length", len(cached)), ("position", n_tokens),
                                                                               ("slot", n_tokens), ("taken", 1))}
    B.page_tables(_ints(cached), _ints(new), t, _ints(free_pages), None if free_at is None else _ints([free_at]), page=page, n_pages=n_pages,
                  n_tokens=n_tokens, offset=None if offset is None else _ints(offset), **out)
    if strided:
        assert bool((buf[:, width:] == 77).all())
    return t.tolist(), out


@pytest.mark.parametrize("seqs,most_new,most_cached,page", [
    (1, 1, 0, 16), (1, 1, 40, 16), (3, 1, 100, 16), (64, 1, 1000, 16), (65, 5, 100, 32), (513, 3, 50, 16), (1000, 130, 300, 16), (7, 3000, 5000, 1024),
    (2, 40000, 3, 64), (8192, 2, 40, 16), (5, 0, 30, 16)])
def test_tables(seqs, most_new, most_cached, page):
    from paper_2604_26334_amd import binding as B
    for seed in range(3):
        cached, new, table, free, n_pages = _tables_case(seed, seqs, most_new, most_cached, page)
        offset = None if seed == 0 else [(i * 7919) % 5000 for i in range(seqs)]
        free_at, n = (None, 0, 3)[seed], sum(new) + seed
        want = O.page_tables(cached, new, table, free, free_at or 0, page, n_pages, n, offset)
        for _ in range(2):       # repeated: the same
            got, out = _run_tables(B, cached, new, table, free, free_at, page, n_pages, n, offset, strided=seed == 1)
            m = want[1][-1]
            assert got == want[0]
            assert out["first"].tolist() == want[1] and out["length"].tolist() == want[2] and out["taken"].tolist() == [want[5]]
            assert out["position"].tolist() == want[3] + [-9] * (n - m) and out["slot"].tolist() == want[4] + [-9] * (n - m)
            table = got


def test_tables_bound_what_they_are_given():
    """A short list of free pages, entries that name no page, tables too narrow, no room for all tokens, lengths out of range."""
    from paper_2604_26334_amd import binding as B
    for seed, kw, room, change in ((0, dict(free=3), None, None), (1, dict(wild=True), None, None), (2, dict(width=3), None, None), (3, {}, 17, None), (4, {}, 0, None),
                                   (5, dict(n_pages=20), None, None), (6, dict(free=0), None, None), (7, {}, 300, "wild")):
        cached, new, table, free, n_pages = _tables_case(seed, 9, 40, 90, 16, **kw)
        if change:
            cached[2], cached[4], cached[5], new[1], new[6], new[8] = -7, 2 ** 31 - 1, 2 ** 30 - 3, -2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1
        for free_at in (0, 2, -4, 2 ** 31 - 1, -2 ** 31):
            n = sum(new) if room is None else room
            want = O.page_tables(cached, new, table, free, free_at, 16, n_pages, n)
            got, out = _run_tables(B, cached, new, table, free, free_at, 16, n_pages, n)
            m = want[1][-1]
            assert got == want[0] and out["first"].tolist() == want[1] and out["length"].tolist() == want[2] and out["taken"].tolist() == [want[5]]
            assert out["position"].tolist() == want[3] + [-9] * (n - m) and out["slot"].tolist() == want[4] + [-9] * (n - m)


# ------------------------------------------------------------------ rows of new tokens

@pytest.mark.parametrize("ty,n,h,d,page,lay", [("f16", 1, 2, 128, 16, "heads"), ("bf16", 65, 8, 128, 32, "heads"), ("f16", 300, 3, 64, 16, "rows"), ("f32", 17, 1, 4, 64, "heads"),
                                               ("f16", 1000, 2, 2048, 16, "rows"), ("bf16", 5000, 4, 80, 128, "rows")])
def test_append(ty, n, h, d, page, lay):
    from paper_2604_26334_amd import binding as B
    torch, g = _t(), _gen(n)
    pages = n // page + 7
    qkv = torch.randn(n, 4, h, d, generator=g, device=DEV).to(_dt(ty))
    shape = (pages, 2, h, page, d) if lay == "heads" else (pages, 2, page, h, d)
    pool = torch.randn(shape, generator=g, device=DEV).to(_dt(ty))
    kp, vp = (pool[:, 0], pool[:, 1]) if lay == "heads" else (pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2))
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:n].to(torch.int32)
    for i, bad in ((1, -1), (3, pages * page), (4, 2 ** 31 - 1), (5, -2 ** 31)):
        if i < n - 1:
            slot[i] = bad
    want = pool.clone()
    wk, wv = (want[:, 0], want[:, 1]) if lay == "heads" else (want[:, 0].transpose(1, 2), want[:, 1].transpose(1, 2))
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < pages * page:
            wk[s // page, :, s % page] = qkv[t, 2]
            wv[s // page, :, s % page] = qkv[t, 3]
    got = B.page_append(qkv[:, 2], qkv[:, 3], kp, vp, slot)
    assert got[0].data_ptr() == kp.data_ptr() and _same_bits(pool, want)


# ------------------------------------------------------------------ attention

def _attend_case(ty, d, hq, hk, page, toks, lens, groups=(), plens=(), seed=0, sharp=1.0, lay="heads", pad=0, holes=False, bound=0):
    """groups: first sequence of each prefix's, then the end.  What no table names, and rows behind a length, hold nan and inf.  bound: of the prefixes,
    by which work is dealt out (prefixes of up to 196608 positions over all sequences and kv heads are walked with the sequences' own positions, longer ones by
    themselves)."""
    torch, g, rng, dt = _t(), _gen(seed + 5), np.random.default_rng(seed), _dt(ty)
    n = sum(toks) + pad
    q = (torch.randn(n, (hq + 2 * hk) * d, generator=g, device=DEV) * sharp).to(dt)[:, :hq * d].view(n, hq, d)
    need = [-(-x // page) for x in list(lens) + list(plens)]
    n_pages = sum(need) + 3
    shape = (n_pages, 2, hk, page, d) if lay == "heads" else (n_pages, 2, page, hk, d)
    pool = torch.randn(shape, generator=g, device=DEV).to(dt)
    kp, vp = (pool[:, 0], pool[:, 1]) if lay == "heads" else (pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2))
    order, tables = [int(x) for x in rng.permutation(n_pages)], []
    used = 0
    for x, m in zip(list(lens) + list(plens), need):
        row = order[used:used + m]
        used += m
        if x % page:                # what lies behind a length is never read
            kp[row[-1], :, x % page:] = float("nan")
            vp[row[-1], :, x % page:] = float("inf")
        if holes:
            row = [int(rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31])) if rng.random() < 0.3 else p for p in row]
        tables.append(row)
    for p in order[used:]:
        kp[p], vp[p] = float("nan"), float("inf")
    b = len(toks)
    wide = [max([len(r) for r in t] + [1]) for t in (tables[:b], tables[b:])]
    full = [[r + [order[-1]] * (w - len(r)) for r in t] for t, w in zip((tables[:b], tables[b:]), wide)]
    first = np.concatenate([[0], np.cumsum(toks)]).astype(int).tolist()
    a = dict(q=q, k_pages=kp, v_pages=vp, first=_ints(first), length=_ints(list(lens)), table=_ints(full[0]), max_length=max(lens), max_tokens=max(toks))
    if plens:
        columns = [order[-1]] * max(0, -(-bound // page) - wide[1])
        a.update(group_first=_ints(list(groups)), prefix_length=_ints(list(plens)), prefix_table=_ints([r + columns for r in full[1]]), max_prefix=max(list(plens) + [bound]))
    return a, first, full


def _check_attend(a, out, first, full, toks, lens, groups, plens, ty, scale=None):
    d, hk = a["q"].shape[2], a["k_pages"].shape[1]
    scale = d ** -0.5 if scale is None else scale
    kp, vp, q = _np(a["k_pages"]), _np(a["v_pages"]), _np(a["q"])
    got = _np(out)
    for s, (t, length) in enumerate(zip(toks, lens)):
        if t == 0:
            continue
        p, pk, pv, pt = 0, np.zeros((hk, 0, d)), np.zeros((hk, 0, d)), np.zeros(0, bool)
        for i, pl in enumerate(plens):
            if groups[i] <= s < groups[i + 1]:
                p, (pk, pt), (pv, _) = pl, O.rows_of(kp, full[1][i], pl), O.rows_of(vp, full[1][i], pl)
        (k, there), (v, _) = O.rows_of(kp, full[0][s], length), O.rows_of(vp, full[0][s], length)
        k, v, there = np.concatenate([pk, k], 1), np.concatenate([pv, v], 1), np.concatenate([pt, there])
        if length < t:              # the first tokens see no own position
            ref = np.zeros((t, q.shape[1], d))
            for i in range(t):
                ref[i] = O.attention(q[first[s] + i:first[s] + i + 1], k, v, there, p + max(-1, length - t + i), scale)[0]
        else:
            ref = O.attention(q[first[s]:first[s] + t], k, v, there, p + length - t, scale)
        seen_k, seen_v = np.where(there[None, :, None], k, 0), np.where(there[None, :, None], v, 0)
        size = np.abs(q[first[s]:first[s] + t]).sum(-1).max() * (np.abs(seen_k).max() if k.size else 0) * abs(scale) * 4
        tol = _attention_tolerance(ref, np.abs(seen_v).max() if v.size else 0, size * (d + 8) / d + 8, ty)
        off = np.abs(got[first[s]:first[s] + t] - ref)
        assert np.isfinite(off).all() and (off <= tol).all(), (s, t, length, p, (off / np.maximum(tol, 1e-30)).max())


ATTEND = [
    # d, q heads, kv heads, page, tokens, own lengths, groups, prefixes
    (128, 4, 2, 16, [1], [1], (), ()), (128, 4, 2, 16, [1], [257], (), ()), (64, 2, 2, 16, [1], [40], (0, 1), [1]),
    (128, 4, 2, 16, [1, 1, 1], [40, 1, 17], (0, 3), [77]), (128, 32, 8, 32, [1] * 9, [i * 37 + 1 for i in range(9)], (0, 9), [300]),
    (64, 16, 2, 64, [1] * 20, [i * 53 % 200 + 1 for i in range(20)], (0, 7, 15), [130, 65]), (128, 8, 8, 128, [1] * 40, [3 + i for i in range(40)], (0, 40), [700]),
    (128, 4, 1, 16, [3, 1, 0, 2], [3, 9, 5, 100], (1, 3), [33]), (64, 8, 2, 16, [8, 5, 1, 8], [8, 64, 65, 300], (0, 2, 4), [31, 32]),
    (128, 4, 4, 16, [33, 40], [40, 333], (0, 2), [100]), (64, 6, 2, 32, [70, 1, 129], [70, 500, 200], (0, 1, 3), [257, 64]),
    (128, 16, 2, 16, [130, 9, 64], [130, 9, 1000], (), ()), (128, 32, 4, 1024, [2] * 33, [900 + i for i in range(33)], (0, 33), [1500]),
    (64, 1, 1, 16, [1] * 130, [i % 90 + 1 for i in range(130)], (0, 129, 130), [16, 48]), (128, 64, 1, 16, [2, 2], [20, 333], (0, 2), [64]),
    (128, 3, 1, 16, [5] * 30, [i * 13 % 90 + 5 for i in range(30)], (0, 10, 10, 25), [50, 9, 200]),
    (64, 8, 2, 128, [60, 200], [60, 700], (0, 2), [300]), (128, 8, 2, 256, [40, 33], [40, 500], (), ()), (64, 4, 4, 1024, [100], [2500], (), ()),
    (128, 6, 2, 64, [7, 2], [90, 64], (0, 1, 2), [128, 640]), (64, 8, 1, 64, [4] * 9, [64 + i for i in range(9)], (0, 5, 9), [64, 129]),
]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention(ty, case, bound):
    from paper_2604_26334_amd import binding as B
    d, hq, hk, page, toks, lens, groups, plens = ATTEND[case]
    a, first, full = _attend_case(ty, d, hq, hk, page, toks, lens, groups, plens, case, sharp=(1.0, 4.0)[case % 2], lay=("heads", "rows")[case // 2 % 2], bound=bound)
    out = B.page_attention(**a)
    _check_attend(a, out, first, full, toks, lens, groups, plens, ty)
    assert _same_bits(out, B.page_attention(**a))


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("d,hq,hk,page,toks,lens,plens", [(128, 32, 8, 16, [1] * 5, [700, 1, 33, 64, 5000], [4097]), (64, 8, 2, 64, [1], [70001], []),
                                                          (128, 8, 2, 32, [24, 24], [300, 24], [9000]), (64, 16, 2, 16, [2] * 17, [50] * 17, [20003]),
                                                          (128, 32, 8, 16, [1] * 24, [1 + 70 * i for i in range(24)], [4097]), (128, 24, 2, 64, [2, 1], [900, 1], [12321])])
def test_attention_over_long_contexts(ty, d, hq, hk, page, toks, lens, plens):
    """Sharp scores; positions at the boundaries of tiles, pages and splits are each some token's favourite."""
    from paper_2604_26334_amd import binding as B
    groups = (0, len(toks)) if plens else ()
    a, first, full = _attend_case(ty, d, hq, hk, page, toks, lens, groups, plens, 3, sharp=3.0)
    for row, length in ((full[1][0], plens[0]) if plens else (full[0][0], lens[0]),):
        for i, p in enumerate([0, 15, 16, 31, 32, 63, 64, 127, 128, 1023, 1024, length // 2, length - 33, length - 1]):
            p = min(max(p, 0), length - 1)
            a["k_pages"][row[p // page], :, p % page] = a["q"][i % len(a["q"]), ::hq // hk] * 0.7
    _check_attend(a, B.page_attention(**a), first, full, toks, lens, groups, plens, ty)


@pytest.mark.parametrize("bound", [0, 1000, 200000])
def test_empty_rows_are_zero(bound):
    """Tokens without a position, sequences of length 0 and prefixes of length 0; pages that name nothing."""
    from paper_2604_26334_amd import binding as B
    for toks, lens, groups, plens in (([1, 2, 3, 1], [0, 1, 2, 5], (), ()), ([2, 3, 1], [0, 1, 3], (0, 1, 3), [0, 40]), ([40, 50], [0, 30], (0, 1), [0]),
                                      ([60, 1], [10, 0], (0, 2), [33]), ([1, 1], [0, 0], (), ())):
        a, first, full = _attend_case("f16", 64, 4, 2, 16, toks, lens, groups, plens, 4, bound=bound)
        out = B.page_attention(**a)
        _check_attend(a, out, first, full, toks, lens, groups, plens, "f16")
        if not plens:
            assert bool((out[:max(0, toks[0] - lens[0])] == 0).all())
    for seed in range(4):
        toks, lens, groups, plens = ([1, 1, 2, 1], [17, 100, 40, 16], (0, 2), [90]) if seed % 2 else ([50, 30], [50, 99], (0, 2), [64])
        a, first, full = _attend_case("f16", 128, 4, 2, 16, toks, lens, groups, plens, seed, holes=True, bound=bound)
        _check_attend(a, B.page_attention(**a), first, full, toks, lens, groups, plens, "f16")
    a["table"].fill_(-1)
    a["prefix_table"].fill_(99999)
    assert bool((B.page_attention(**a) == 0).all())


@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("hq,toks", [(4, [1, 3, 8]), (16, [2, 1, 4]), (4, [40, 3, 70])])
def test_hidden_positions_may_hold_anything(hq, toks, bound):
    """A position that a token does not see does not count, whatever its key and value hold; one that it sees does."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    lens = [t + 20 for t in toks]
    a, first, full = _attend_case("f16", 128, hq, 2, 16, toks, lens, (0, 2), [50], 6, bound=bound)
    clean = B.page_attention(**a)
    p = lens[2] - toks[2] // 2                 # an own position of the last sequence in the middle of its new tokens
    i = p - (lens[2] - toks[2])                # the first token that sees it
    for bad in (float("nan"), float("inf"), -65504.0):
        for key in (True, False):
            k, v = a["k_pages"].clone(), a["v_pages"].clone()
            (k if key else v)[full[0][2][p // 16], :, p % 16] = bad
            out = B.page_attention(**dict(a, k_pages=k, v_pages=v))
            assert _same_bits(out[:first[2] + i], clean[:first[2] + i])
            if bad != -65504.0 and not key:
                assert not bool(torch.isfinite(out[first[2] + i:]).any())
            if bad != bad:
                assert not bool(torch.isfinite(out[first[2] + i:]).any())


@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("toks", [[1, 1, 1], [2] * 20, [60, 9]])
def test_keys_that_are_no_numbers_reach_every_token_that_sees_them(toks, bound):
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for where in ("prefix", "own"):
        for lo, hi in ((0, 16), (0, 64), (64, 192), (0, 400), (384, 400)):
            a, first, full = _attend_case("f16", 64, 4, 2, 16, toks, [400 + t for t in toks], (0, len(toks)), [400], 3, bound=bound)
            for i in range(lo, hi):
                row = full[1][0] if where == "prefix" else full[0][0]
                a["k_pages"][row[i // 16], 1, i % 16] = float("nan")
            fine = torch.isfinite(B.page_attention(**a)).all(-1)
            rows = len(fine) if where == "prefix" else toks[0]
            assert bool(fine[:, :2].all()) and not bool(fine[:rows, 2:].any()) and bool(fine[rows:].all()), (where, lo, hi)


@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("toks", [[1, 2], [40, 3]])
@pytest.mark.parametrize("scale", [-0.09, 0.0, 1.3])
def test_attention_with_any_scale(toks, scale, bound):
    from paper_2604_26334_amd import binding as B
    a, first, full = _attend_case("bf16", 128, 4, 2, 16, toks, [333, 40], (0, 2), [99], 6, bound=bound)
    _check_attend(a, B.page_attention(**a, scale=scale), first, full, toks, [333, 40], (0, 2), [99], "bf16", scale)


@pytest.mark.parametrize("bound", [0, 1000, 200000])
def test_attention_of_padded_batches_and_bounded_values(bound):
    """Rows behind the last sequence keep what they hold; lengths, offsets and groups out of range are bounded as documented."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    toks, lens, groups, plens = [5, 0, 4], [20, 3, 30], (0, 2), [70]
    a, first, full = _attend_case("f16", 128, 4, 2, 16, toks, lens, groups, plens, 5, pad=7, bound=bound)
    out = torch.full((16, 4, 128), 3.0, dtype=torch.float16, device=DEV)
    B.page_attention(**a, out=out)
    _check_attend(a, out, first, full, toks, lens, groups, plens, "f16")
    assert bool((out[9:] == 3).all())
    # longer ones count as their bounds, negative ones as none; tokens beyond max_tokens are left out
    out.fill_(3.0)
    b = dict(a, length=_ints([2 ** 31 - 1, 0, -5]), prefix_length=_ints([2 ** 31 - 1]), max_length=19, max_prefix=33, max_tokens=4)
    b["k_pages"], b["v_pages"] = (torch.where(torch.isfinite(a[n]), a[n], 0.5) for n in ("k_pages", "v_pages"))
    B.page_attention(**b, out=out)
    # (the first of five tokens sees 19 - 5 + 1 positions; the fifth is not answered)
    want = torch.full_like(out, 3.0)
    B.page_attention(**dict(b, length=_ints([19, 0, 0]), prefix_length=_ints([33]), max_tokens=5, max_prefix=a["max_prefix"]), out=want)
    assert bool((out[4] == 3).all()) and bool((out[9:] == 3).all())
    err = (out[:4].float() - want[:4].float()).abs().max()
    # (two results, each off by half a step of a value up to 5 and of the values' spread, up to 10, and by fp32's sums: 32 half steps)
    assert float(err) <= 32 * 2.0 ** -11 and bool((out[5:9] == 0).all())
    # offsets and groups: bounded; a sequence that ends before it starts has no token
    out.fill_(3.0)
    B.page_attention(**dict(b, first=_ints([12, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]), group_first=_ints([-7, 2 ** 31 - 1])), out=out)
    assert bool((out[:12] == 3).all()) and bool(torch.isfinite(out).all()) and not bool((out[12:] == 3).all())
    out.fill_(3.0)
    for n in ("group_first", "prefix_length", "prefix_table"):
        b[n] = None
    B.page_attention(**dict(b, first=_ints([12, 2 ** 31 - 1, 7, -3])), out=out)
    assert bool((out[:12] == 3).all()) and bool(torch.isfinite(out).all())


def test_attention_without_positions_needs_no_tables():
    """max_length 0, or a pool of no pages: zeros, whatever the tables are."""
    import ctypes as C
    from paper_2604_26334_amd import binding as B
    torch = _t()
    q = torch.ones(3, 4, 64, dtype=torch.float16, device=DEV)
    first, length, pages = _ints([0, 1, 3]), _ints([5, 7]), torch.full((2, 2, 16, 64), float("nan"), dtype=torch.float16, device=DEV)
    gf, pl = _ints([0, 2]), _ints([20])
    for kw in (dict(max_length=0, n_pages=2, k_pages=pages.data_ptr(), v_pages=pages.data_ptr()), dict(max_length=128, n_pages=0),
               dict(max_length=0, n_pages=0, n_prefix=1, prefix_width=4, max_prefix=64, group_first=gf.data_ptr(), prefix_length=pl.data_ptr()),
               dict(max_length=0, n_pages=2, k_pages=pages.data_ptr(), v_pages=pages.data_ptr(), n_prefix=1, prefix_width=4, max_prefix=0,
                    group_first=gf.data_ptr(), prefix_length=pl.data_ptr())):
        for tokens in (2, 40):
            out = torch.full_like(q, 3.0)
            a = B.ps_page_attention_args(type=0, n_seq=2, n_tokens=3, n_q_heads=4, n_kv_heads=2, head_dim=64, page=16, width=8, max_tokens=tokens, scale=0.1,
                                         q=q.data_ptr(), out=out.data_ptr(), q_token=256, q_head=64, out_token=256, out_head=64, k_page=2048, k_head=1024, k_row=64,
                                         v_page=2048, v_head=1024, v_row=64, table_seq=8, prefix_seq=4, first=first.data_ptr(), length=length.data_ptr(), **kw)
            need = C.c_uint64()
            assert B.lib().ps_page_attention_workspace(C.byref(a), C.byref(need)) == 0
            work = torch.empty(need.value + 1, dtype=torch.uint8, device=DEV)
            assert B.lib().ps_page_attention(C.byref(a), work.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
            assert bool((out == 0).all()), kw


def test_attention_far_into_a_large_pool():
    """Offsets past 32 bits: pages 2^25 elements apart, 300 of them."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    step, pages = 1 << 25, 130
    far = torch.empty(pages * step, dtype=torch.float16, device=DEV).as_strided((pages, 2, 2, 16, 64), (step, 2048, 1024, 64, 1))
    for toks, lens, groups, plens in (([1, 1, 2], [700, 33, 400], (0, 2), [600]), ([50, 3], [300, 800], (0, 2), [500])):
        a, first, full = _attend_case("f16", 64, 4, 2, 16, toks, lens, groups, plens, 8)
        n = a["k_pages"].shape[0]
        assert n <= pages
        far[:n, 0], far[:n, 1] = a["k_pages"], a["v_pages"]
        assert _same_bits(B.page_attention(**a), B.page_attention(**dict(a, k_pages=far[:n, 0], v_pages=far[:n, 1])))
        # the last pages, whose offsets are past 2^32 bytes and elements alike
        shift = pages - n
        far[shift:, 0], far[shift:, 1] = a["k_pages"].clone(), a["v_pages"].clone()
        b = dict(a, k_pages=far[:, 0], v_pages=far[:, 1], table=a["table"] + shift, prefix_table=a["prefix_table"] + shift)
        assert _same_bits(B.page_attention(**a), B.page_attention(**b))
        k = torch.randn(sum(toks), 2, 64, generator=_gen(3), device=DEV).half()
        slot = _ints([pages * 16 - 1 - i for i in range(sum(toks))])
        B.page_append(k, k, far[:, 0], far[:, 1], slot)
        for i in range(sum(toks)):
            assert _same_bits(far[-1 - i // 16, 0, :, 15 - i % 16], k[i])


# ------------------------------------------------------------------ sampling

def _check_sample(logits, u, token, kept, temperature=None, top_k=None, top_p=None, min_p=None):
    """The oracle's sums are right to V 2^-53 (2^-29 at 2^24 entries), the kernel's to 2e-11 of each weight: a border that lies closer to its
    goal than 1e-10 of the sum (2^-28 where a vocabulary passes 2^17) may be passed one entry earlier or later."""
    for i, x in enumerate(_np(logits)):
        s = dict(temperature=1.0 if temperature is None else float(temperature[i]), top_k=0 if top_k is None else int(top_k[i]),
                 top_p=1.0 if top_p is None else float(top_p[i]), min_p=0.0 if min_p is None else float(min_p[i]))
        at, total, n = O.kept(x, **s)
        want = O.sample(x, float(u[i]), **s)
        got = (int(token[i]), int(kept[i]))
        if got == want:
            continue
        assert n and got[1] >= 1, (i, s, got, want)
        near = (1e-10 if len(x) <= 1 << 17 else 2.0 ** -28) * total[-1]
        if got[1] != n:          # a border of top-p, or a weight on the border of min-p
            goal = s["top_p"] * total[min(s["top_k"] if s["top_k"] > 0 else len(total), len(total)) - 1]
            lo, hi = sorted((n, got[1]))
            w = np.diff(np.concatenate([[0.0], total]))
            assert (np.abs(total[lo - 1:hi] - goal) <= near).any() or (np.abs(w[lo - 1:hi + 1] - s["min_p"]) <= 1e-10).any(), (i, s, got, want)
        r = int(np.flatnonzero(at == got[0])[0])
        goal = float(u[i]) * total[got[1] - 1]
        assert r < got[1] and total[r] > goal - near and (r == 0 or total[r - 1] <= goal + near), (i, s, got, want)


SETTINGS = [dict(), dict(top_k=True), dict(top_p=True), dict(min_p=True), dict(top_k=True, top_p=True, min_p=True), dict(temperature=True, top_k=True, top_p=True)]


def _settings(rng, n, V, which):
    torch = _t()
    s = {}
    if which.get("temperature"):
        s["temperature"] = rng.choice([0.0, 0.05, 0.7, 1.0, 1.5, 100.0, -1.0, float("nan"), float("inf")], n)
    if which.get("top_k"):
        s["top_k"] = rng.choice([1, 2, 5, 50, 1000, 0, -3, V - 1, V, V + 1, 2 ** 31 - 1], n)
    if which.get("top_p"):
        s["top_p"] = rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 0.9999, 1.0, 1.5, -1.0, float("nan")], n)
    if which.get("min_p"):
        s["min_p"] = rng.choice([0.0, 0.001, 0.05, 0.3, 1.0, 2.0, -1.0, float("nan")], n)
    return {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) for k, v in s.items()}


@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("which", range(len(SETTINGS)))
@pytest.mark.parametrize("n,V,spread", [(1, 1, 1.0), (3, 2, 1.0), (9, 7, 3.0), (24, 1000, 2.5), (40, 257, 0.0), (12, 32000, 2.5), (5, 32001, 0.1), (6, 128256, 2.5), (3, 128256, 40.0), (4, 128256, 0.0), (4, 70000, 0.01), (3, 32768, 1.0), (3, 32769, 1.0)])
def test_sample(ty, which, n, V, spread):
    from paper_2604_26334_amd import binding as B
    torch, g = _t(), _gen(V + which)
    rng = np.random.default_rng(V + which)
    buf = (torch.randn(n, V + 3, generator=g, device=DEV) * spread).to(_dt(ty))
    logits = buf[:, 1:V + 1]                   # rows that start anywhere
    u = torch.tensor([(0.0, 1 - 2.0 ** -24)[i] if i < 2 and n > 2 else x for i, x in enumerate(rng.random(n) * (1 - 2.0 ** -24))], dtype=torch.float32, device=DEV)
    s = _settings(rng, n, V, SETTINGS[which])
    token, kept = B.sample(logits, u, **s)
    _check_sample(logits, u, token, kept, **s)
    again = B.sample(logits.contiguous(), u, **s)
    assert torch.equal(token, again[0]) and torch.equal(kept, again[1])
    # a row by itself, and in a wider type: the same
    wide = B.sample(logits[n // 2:n // 2 + 1].float(), u[n // 2:n // 2 + 1].contiguous(), **{k: v[n // 2:n // 2 + 1].contiguous() for k, v in s.items()})
    assert int(wide[0]) == int(token[n // 2]) and int(wide[1]) == int(kept[n // 2])


def test_sample_draws_every_kept_entry_with_its_share():
    """Random numbers at the borders of the running sum: weights that are powers of two, so every sum is exact."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    x = torch.tensor([-3.0, -1.0, -4.0, -2.0, -4.0], device=DEV)      # in order: entries 1, 3, 0, 2, 4
    T = torch.tensor([1 / np.log(2.0)], dtype=torch.float32, device=DEV)      # weights 2^-e but for the rounding of T, 2^-25 e
    borders = np.cumsum([0.5, 0.25, 0.125, 0.0625, 0.0625])
    for r, b in enumerate(borders[:-1]):
        for step, want in ((-1e-6, [1, 3, 0, 2][r]), (1e-6, [3, 0, 2, 4][r])):
            u = torch.tensor([b + step], dtype=torch.float32, device=DEV)
            token, kept = B.sample(x[None], u, temperature=T)
            assert int(token) == want and int(kept) == 5, (r, step)
    # equal logits: shares of 1 / V, exactly, and top-p takes the lowest indices
    for V in (4, 64, 4096):
        x = torch.full((V, V), 3.25, device=DEV)
        u = torch.arange(V, device=DEV) / V
        assert torch.equal(B.sample(x, u)[0].long(), torch.arange(V, device=DEV))
        token, kept = B.sample(x, torch.full((V,), 1 - 2.0 ** -24, device=DEV), top_p=torch.full((V,), 0.5, device=DEV))
        assert bool((kept == V // 2).all()) and bool((token == V // 2 - 1).all())


def test_sample_random_numbers_out_of_range():
    """Below 0 counts as 0, anything else that is not in [0, 1) as the largest number that is."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for V in (300, 50000):
        x = torch.randn(6, V, generator=_gen(V), device=DEV)
        x[:] = x[0]
        u = torch.tensor([0.0, -3.0, 1 - 2.0 ** -24, 1.0, float("inf"), float("nan")], device=DEV)
        for s in (dict(), dict(top_k=_ints([20] * 6)), dict(top_p=torch.full((6,), 0.5, device=DEV))):
            token, kept = B.sample(x, u, **s)
            assert token.tolist() == [int(token[0])] * 2 + [int(token[2])] * 4 and len(set(kept.tolist())) == 1
            _check_sample(x[:3], u.clamp(0, 1 - 2.0 ** -24)[:3], token[:3], kept[:3], **{k: v[:3] for k, v in s.items()})


def test_calls_at_once_on_streams_of_their_own():
    """Two batches on two streams, several times: each gives what it gives alone."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    work = []
    for i, (toks, lens, groups, plens) in enumerate((([1] * 30, [60 * j + 1 for j in range(30)], (0, 30), [3000]), ([70, 3], [900, 500], (0, 2), [1000]))):
        a, _, _ = _attend_case("f16", 128, 8, 2, 16, toks, lens, groups, plens, i)
        x, u = (torch.randn(9, 90000, generator=_gen(i), device=DEV) * 2).half(), torch.rand(9, generator=_gen(i), device=DEV)
        work.append((a, x, u, B.page_attention(**a), B.sample(x, u, top_p=torch.full((9,), 0.9, device=DEV))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = []
    for _ in range(4):
        for st, (a, x, u, _, _) in zip(streams, work):
            with torch.cuda.stream(st):
                got.append((B.page_attention(**a), B.sample(x, u, top_p=torch.full((9,), 0.9, device=DEV))))
    torch.cuda.synchronize()
    for i, (out, (token, kept)) in enumerate(got):
        want = work[i % 2]
        assert _same_bits(out, want[3]) and torch.equal(token, want[4][0]) and torch.equal(kept, want[4][1]), i


def test_a_workspace_may_hold_anything():
    """What a workspace holds before a call does not show in the results, and nothing behind the bytes that were asked for is written."""
    import ctypes as C
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for toks, lens, groups, plens, bound in (([1, 2, 1] * 5, [700, 33, 1] * 5, (0, 9, 15), [900, 40], 0), ([3] * 4, [50, 3, 900, 2000], (0, 2), [70], 1000),
                                             ([60, 2], [60, 3000], (0, 1), [500], 0), ([1] * 9, [0] * 9, (3, 6), [600], 0)):
        a, _, _ = _attend_case("f16", 64, 8, 2, 16, toks, lens, groups, plens, 7, bound=bound)
        want = B.page_attention(**a)
        for fill in (0, 255, 127):
            work = torch.full((1 << 26,), fill, dtype=torch.uint8, device=DEV)
            assert _same_bits(B.page_attention(**a, workspace=work), want)
    for n, V in ((7, 3000), (5, 90000)):
        x, u = (torch.randn(n, V, generator=_gen(V), device=DEV) * 2).half(), torch.rand(n, generator=_gen(V), device=DEV)
        x[1], x[2] = float("-inf"), 1.0
        s = dict(temperature=torch.tensor([1.0, 1.0, 1.0, 0.0, 0.5] + [2.0] * (n - 5), device=DEV), top_p=torch.full((n,), 0.9, device=DEV), top_k=_ints([100] * n))
        want = B.sample(x, u, **s)
        need = C.c_uint64()
        assert B.lib().ps_sample_workspace(C.byref(B.ps_sample_args(type=0, n_rows=n, vocab=V)), C.byref(need)) == 0
        for fill in (0, 255, 127):
            work = torch.full((need.value + 4096,), fill, dtype=torch.uint8, device=DEV)
            got = B.sample(x, u, **s, workspace=work)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((work[need.value:] == fill).all())


def test_attention_into_a_part_of_a_larger_tensor():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    for toks, lens in (([1, 2, 1], [50, 300, 7]), ([50, 20], [70, 300])):
        a, _, _ = _attend_case("bf16", 64, 8, 2, 32, toks, lens, (0, 2), [100], 2)
        plain = B.page_attention(**a)
        n = plain.shape[0]
        big = torch.full((n, 3, 8, 72), 5.0, dtype=torch.bfloat16, device=DEV)
        out = big[:, 1, :, :64]
        B.page_attention(**a, out=out)
        assert _same_bits(out, plain)
        big[:, 1, :, :64] = 5.0
        assert bool((big == 5).all())


def test_sample_infinities_and_masks():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    inf, nan = float("inf"), float("nan")
    for ty in ("f16", "bf16", "f32"):
        low = torch.finfo(_dt(ty)).min
        rows = [[-inf] * 6, [nan] * 6, [-inf, -inf, 2.0, -inf, nan, -inf], [0.0, inf, 1.0, inf, nan, 2.0], [low] * 6, [low, 1.0, low, 1.0, low, -inf],
                [-0.0, 0.0, -0.0, -inf, 0.0, -0.0], [nan, -inf, low, -inf, nan, -inf]]
        x = torch.tensor(rows, device=DEV).to(_dt(ty))
        for us in (0.0, 0.3, 0.6, 1 - 2.0 ** -24):
            u = torch.full((len(rows),), us, device=DEV)
            for s in (dict(), dict(temperature=torch.zeros(len(rows), device=DEV)), dict(top_k=_ints([2] * len(rows))), dict(top_p=torch.full((len(rows),), 0.7, device=DEV)),
                      dict(min_p=torch.full((len(rows),), 0.5, device=DEV))):
                token, kept = B.sample(x, u, **s)
                _check_sample(x, u, token, kept, **s)
                assert token[:2].tolist() == [-1, -1] and kept[:2].tolist() == [0, 0] and token[2:].min() >= 0


def test_sample_the_largest_vocabulary_and_rows_far_apart():
    from paper_2604_26334_amd import binding as B
    torch = _t()
    V = 1 << 24
    x = torch.randn(2, V, generator=_gen(1), device=DEV) * 2
    for s in (dict(), dict(top_p=torch.tensor([0.9, 0.5], device=DEV)), dict(top_k=_ints([100000, 7]))):
        u = torch.tensor([0.77, 0.2], device=DEV)
        token, kept = B.sample(x, u, **s)
        _check_sample(x, u, token, kept, **s)
    n, step = 300, 1 << 24
    far = torch.empty(n * step, dtype=torch.float16, device=DEV).as_strided((n, 5000), (step, 1))
    near = (torch.randn(n, 5000, generator=_gen(2), device=DEV) * 2.5).half()
    far.copy_(near)
    u = torch.rand(n, generator=_gen(3), device=DEV)
    for a, b in zip(B.sample(far, u, top_p=torch.full((n,), 0.9, device=DEV)), B.sample(near, u, top_p=torch.full((n,), 0.9, device=DEV))):
        assert torch.equal(a, b)


# ------------------------------------------------------------------ a step of all four

def _step_case(seed, b=6, prefix=50, page=16):
    torch, g, rng = _t(), _gen(seed), np.random.default_rng(seed)
    hq, hk, d, V = 4, 2, 64, 300
    cached = [int(rng.integers(0, 60)) for _ in range(b)]
    new = [int(rng.integers(1, 5)) for _ in range(b)]
    width = 6
    pages = b * width + 8
    order = [int(x) for x in rng.permutation(pages)]
    np_pages = -(-prefix // page)
    ptable, at, table = [order[:np_pages]], np_pages, []
    for c in cached:
        h = -(-c // page)
        table.append(order[at:at + h] + [-1] * (width - h))
        at += h
    n = 4 * b
    a = dict(cached=_ints(cached), new=_ints(new), table=_ints(table), free=_ints((order[at:] + [-1] * pages)[:pages]), free_at=_ints([1]), offset=_ints([prefix] * 4 + [0] * (b - 4)),
             group_first=_ints([0, 4]), prefix_length=_ints([prefix]), prefix_table=_ints(ptable), pool=torch.randn(pages, 2, hk, page, d, generator=g, device=DEV).half(),
             q0=torch.randn(n, hq, d, generator=g, device=DEV).half(), k0=torch.randn(n, hk, d, generator=g, device=DEV).half(),
             v=torch.randn(n, hk, d, generator=g, device=DEV).half(), inv_freq=torch.tensor(np.exp(-np.arange(d // 2) / (d // 2) * np.log(10000.0)), dtype=torch.float32, device=DEV),
             head=torch.randn(hq * d, V, generator=g, device=DEV) * 0.3, u=torch.rand(b, generator=g, device=DEV), top_p=torch.full((b,), 0.9, device=DEV),
             temperature=torch.full((b,), 0.8, device=DEV), n=n, pages=pages, page=page)
    return a


def _step(a, B):
    torch = _t()
    first, length, position, slot, taken = B.page_tables(a["cached"], a["new"], a["table"], a["free"], a["free_at"], page=a["page"], n_pages=a["pages"], n_tokens=a["n"],
                                                         offset=a["offset"], position=torch.zeros(a["n"], dtype=torch.int32, device=DEV),
                                                         slot=torch.full((a["n"],), -1, dtype=torch.int32, device=DEV))
    q, k = B.qk_norm_rope(a["q0"], a["k0"], position, a["inv_freq"])
    B.page_append(k, a["v"], a["pool"][:, 0], a["pool"][:, 1], slot)
    out = torch.zeros_like(q)
    B.page_attention(q, a["pool"][:, 0], a["pool"][:, 1], first, length, a["table"], max_length=96, max_tokens=4, group_first=a["group_first"],
                     prefix_length=a["prefix_length"], prefix_table=a["prefix_table"], max_prefix=64, out=out)
    last = out.view(a["n"], -1)[(first[1:] - 1).long()].float()
    logits = (last[:, :, None] * a["head"]).sum(1).half()
    token, kept = B.sample(logits, a["u"], temperature=a["temperature"], top_p=a["top_p"])
    return first, length, position, slot, taken, q, k, out, logits, token, kept


def test_a_step_of_all_four():
    from oracle import drafts as D
    from paper_2604_26334_amd import binding as B
    a = _step_case(1)
    pool0, table0 = a["pool"].clone(), a["table"].tolist()
    first, length, position, slot, taken, q, k, out, logits, token, kept = _step(a, B)
    want = O.page_tables(a["cached"].tolist(), a["new"].tolist(), table0, a["free"].tolist(), 1, 16, a["pages"], a["n"], a["offset"].tolist())
    m = want[1][-1]
    assert a["table"].tolist() == want[0] and first.tolist() == want[1] and length.tolist() == want[2] and position.tolist()[:m] == want[3] and slot.tolist()[:m] == want[4]
    qr, kr = (D.qk_norm_rope(_np(a[x])[:m], None, want[3], a["inv_freq"].cpu().numpy(), 1e-6, True, False) for x in ("q0", "k0"))
    pool = _np(pool0)
    for t, s in enumerate(want[4]):
        pool[s // 16, 0, :, s % 16], pool[s // 16, 1, :, s % 16] = kr[t], _np(a["v"])[t]
    assert np.abs(_np(a["pool"]) - pool).max() <= np.abs(kr).max() * 2.0 ** -10
    for s, n in enumerate(a["new"].tolist()):
        (k1, there), (v1, _) = O.rows_of(pool[:, 0], want[0][s], want[2][s]), O.rows_of(pool[:, 1], want[0][s], want[2][s])
        p = 0
        if s < 4:
            (pk, pt), (pv, _) = O.rows_of(pool[:, 0], a["prefix_table"].tolist()[0], 50), O.rows_of(pool[:, 1], a["prefix_table"].tolist()[0], 50)
            k1, v1, there, p = np.concatenate([pk, k1], 1), np.concatenate([pv, v1], 1), np.concatenate([pt, there]), 50
        r = slice(want[1][s], want[1][s + 1])
        ref = O.attention(qr[r], k1, v1, there, p + want[2][s] - n, 64 ** -0.5)
        # queries and keys are rounded to fp16 in between (2^-11 each, scores of up to about 20: 0.02 of a weight)
        assert np.abs(_np(out[r]) - ref).max() < 0.02 * np.abs(ref).max() * 4
    _check_sample(logits, a["u"], token, kept, temperature=a["temperature"], top_p=a["top_p"])


def test_a_step_on_another_stream_and_replayed():
    """The four as one captured graph, on a stream of its own: every replay gives the eager call's bits, with eager calls and other inputs in between."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    a = _step_case(2)
    pool0, table0 = a["pool"].clone(), a["table"].clone()
    want = [t.clone() for t in _step(a, B)] + [a["pool"].clone(), a["table"].clone()]
    other = _step_case(3)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a["pool"].copy_(pool0)
        a["table"].copy_(table0)
        got = _step(a, B)
        stream.synchronize()
        for x, y in zip(list(got) + [a["pool"], a["table"]], want):
            assert _same_bits(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = _step(a, B)
    for i in range(4):
        a["pool"].copy_(pool0)
        a["table"].copy_(table0)
        for t in res:
            t.zero_()
        _step(other, B)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(list(res) + [a["pool"], a["table"]], want):
            assert _same_bits(x, y), i
    # other requests in the same places
    fresh = _step_case(3)
    for name in ("q0", "k0", "v", "u", "cached", "new", "table", "free", "offset", "pool"):
        a[name].copy_(fresh[name])
    pool0, table0 = a["pool"].clone(), a["table"].clone()
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in res] + [a["pool"].clone(), a["table"].clone()]
    a["pool"].copy_(pool0)
    a["table"].copy_(table0)
    for x, y in zip(list(_step(a, B)) + [a["pool"], a["table"]], replayed):
        assert _same_bits(x, y)


@pytest.mark.parametrize("mode", [0, 1])
def test_a_stacks_next_tokens(mode):
    """A stack's logits, drawn from on its compute stream behind each forward, without a wait between them."""
    import synth_inputs as S
    from paper_2604_26334_amd import binding as B
    from tests import harness as Hn
    from tests.test_gpu_head import _budgets, _load_all
    torch = _t()
    M, V = 16, 1040
    cfg = dict(Hn.small_dense_cfg(2), vocab=V)
    plan = B.Plan(cfg, _budgets(cfg, M, [1.0])[0], M)
    st = B.Stack(plan)
    st.set_decode_mode(mode)
    _load_all(st, cfg, Hn.WeightCache(cfg, 9), S.head_matrix(9, cfg))
    xin = torch.from_numpy(np.ascontiguousarray(S.activations(9, 0, M, cfg["hidden"]))).to(st.device)
    xout, logits = torch.empty_like(xin), torch.full((M, V), 7.0, dtype=torch.float16, device=st.device)
    u = torch.rand(M, generator=_gen(1), device=DEV)
    s = dict(temperature=torch.full((M,), 0.8, device=DEV), top_k=_ints([40] * M), top_p=torch.full((M,), 0.95, device=DEV))
    st.set_logits_out(logits, 0, M)
    torch.cuda.synchronize()
    for _ in range(3):
        st.forward(xin, xout)
        with torch.cuda.stream(st.compute):
            token, kept = B.sample(logits, u, **s)
        st.synchronize()
        _check_sample(logits, u, token, kept, **s)
        assert int(kept.max()) <= 40 and len(set(token.tolist())) > 1
    st.close()
    plan.close()
