"""Operators of a batch of requests at the ends of their ranges."""
import numpy as np
import pytest

from oracle import batch as O
from oracle import drafts as D
from tests import test_gpu_batch as T
from tests import test_gpu_batch_weights as W
from tests.test_gpu_drafts import DEV, _dt, _gen, _half_step, _ints, _np, _same_bits, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cached,new", [
    ([0, 5], [2 ** 30, 2 ** 30]), ([2 ** 30, 2 ** 30, 7, 2 ** 30], [2 ** 29] * 4), ([3] * 70, [2 ** 31 - 1] * 70), ([2 ** 31 - 1, 2 ** 30 - 1], [1, 2 ** 30]),
    ([0] * 600, [2 ** 21 + 1] * 600), ([1, 2, 3], [2 ** 30 - 2, 1, 5])])
def test_tables_of_as_many_tokens_as_there_may_be(cached, new):
    """n_tokens of 2^30, and new tokens that come to it or to more: their sums end there, and nothing behind the arrays is written."""
    from paper_2604_26334_amd import binding as B
    torch, n, guard, page, width = _t(), 1 << 30, 1 << 20, 1024, 2
    seqs = len(cached)
    buf = torch.full((2, n + guard), -9, dtype=torch.int32, device=DEV)
    table, free = torch.full((seqs, width), 3, dtype=torch.int32, device=DEV), torch.arange(100, 100 + 2 * seqs, dtype=torch.int32, device=DEV)
    first, length, position, slot, taken = B.page_tables(_ints(cached), _ints(new), table, free, None, page=page, n_pages=5000, n_tokens=n, position=buf[0, :n],
                                                         slot=buf[1, :n])
    want_first, want_length, pages, rows = [0], [], 0, [[3] * width for _ in range(seqs)]
    for s in range(seqs):
        c = min(cached[s], 2 ** 30)
        t = min(new[s], n - want_first[-1])
        want_first.append(want_first[-1] + t)
        want_length.append(min(c + t, 2 ** 30))
        for entry in range(min(width, -(-c // page)), min(width, -(-want_length[-1] // page))):
            rows[s][entry] = 100 + pages
            pages += 1
    assert first.tolist() == want_first and length.tolist() == want_length and int(taken) == pages and table.tolist() == rows
    total = want_first[-1]
    assert bool((buf[:, total:] == -9).all())
    at = np.unique(np.concatenate([np.clip(np.array(want_first)[:, None] + np.arange(-3, 2051), 0, total - 1).ravel(), np.linspace(0, total - 1, 1001).astype(np.int64)]))
    s = np.searchsorted(np.array(want_first[1:]), at, side="right")
    j = np.minimum(np.array(cached), 2 ** 30)[s] + at - np.array(want_first)[s]
    there = torch.from_numpy(at).to(DEV)
    assert np.array_equal(position[there].cpu().numpy(), j.astype(np.int32))
    entry = np.minimum(j // page, width - 1)
    assert np.array_equal(slot[there].cpu().numpy(), np.where(j // page < width, np.array(rows)[s, entry] * page + j % page, -1))


# Scores of 2^29 and of 64 more: neighbours among fp32's numbers there, 8 nats apart at a scale of 1/8.  Sums of two products each, which are exact.
LARGE = 2.0 ** 29


def _large_scores(ty, n, t, d, heads):
    """Queries [t, heads, d] and keys [n, d] of which the first 16 positions score 2^29, two in each later tile 2^29 + 64 and all others 0"""
    torch = _t()
    q, k = torch.zeros(t, heads, d, dtype=_dt(ty), device=DEV), torch.zeros(n, d, dtype=_dt(ty), device=DEV)
    q[..., 0], q[..., 1] = 16384.0, 8.0
    k[:16, 0] = 32768.0
    for p in range(128, n, 16):
        k[p + 2, 0], k[p + 2, 1] = 32768.0, 8.0
    return q, k, torch.randn(n, d, generator=_gen(n), device=DEV).to(_dt(ty))


def _near_weights(out, ref, v, ty):
    """Half a step of the result, and of the weights against their sum (the spread of the values each); the exponential's argument, up to 12 in powers of two, and
    the exponential in fp32: less than 2^-19 of a weight."""
    off = np.abs(_np(out) - ref)
    assert np.isfinite(_np(out)).all()
    assert (off <= np.abs(ref) * _half_step(ty) + 2 * np.abs(_np(v)).max() * (_half_step(ty) + 2.0 ** -19)).all(), off.max()


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("bound", [0, 200000])
@pytest.mark.parametrize("d,t,prefix", [(64, 1, 0), (128, 2, 0), (128, 20, 0), (64, 40, 0), (128, 1, 400), (64, 20, 400), (128, 40, 400)])
def test_large_scores_next_to_each_other(ty, bound, d, t, prefix):
    """Weights stay in their type's range however large the scores are.  512 heads, so that no run ends between the two kinds of keys."""
    torch = _t()
    q, k, v = _large_scores(ty, 400, t, d, 512)
    k, v = (torch.cat((x, torch.zeros(t, d, dtype=x.dtype, device=DEV))) for x in (k, v))
    ref = O.attention(_np(q[:, :1]), _np(k)[None], _np(v)[None], np.ones(400 + t, bool), 400, 0.125)
    _near_weights(W._call(q, k, v, prefix, 0.125, bound), ref, v, ty)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("d,t", [(64, 1), (128, 20), (64, 40)])
def test_large_scores_next_to_each_other_behind_a_tree(ty, d, t):
    from paper_2604_26334_amd import binding as B
    torch = _t()
    q, k, v = _large_scores(ty, 400, t, d, 512)
    new = torch.zeros(t, 1, d, dtype=_dt(ty), device=DEV)
    out = B.tree_attention(q, new.expand(t, 512, d), new.expand(t, 512, d), k.expand(1, 512, 400, d), v.expand(1, 512, 400, d), _ints([0, t]), _ints([400]),
                           _ints([-1] + [0] * (t - 1)), max_context=400, max_tree=t, scale=0.125)
    ref = D.tree_attention(_np(q[:, :1]), _np(new), _np(new), _np(k)[None], _np(v)[None], 400, [-1] + [0] * (t - 1), 0.125)
    _near_weights(out, ref, v, ty)


# sequences' tokens, own lengths, groups, prefixes
ROOM = [([1] * 64, [1 + 7 * i for i in range(64)], (0, 64), [900]), ([2] * 30, [2 + 31 * i for i in range(30)], (0, 9, 25), [300, 77]), ([1], [5000], (), ()),
        ([4] * 9, [300] * 9, (0, 9), [200]), ([40] * 3, [40, 700, 300], (0, 2), [130]), ([1] * 5, [900] * 5, (), ())]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("case", range(len(ROOM)))
def test_room_for_more_tokens_changes_nothing(ty, bound, case):
    """Rows behind the last sequence, however many: the same bits, in the same workspace, and these rows as they were."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    toks, lens, groups, plens = ROOM[case]
    a, first, full = T._attend_case(ty, 128, 8, 2, 16, toks, lens, groups, plens, case, bound=bound)
    want = B.page_attention(**a)
    T._check_attend(a, want, first, full, toks, lens, groups, plens, ty)
    n = sum(toks)
    for pad, at in ((1, 0), (1000, 0), (1000, 37), (20000, 19999)):             # (the first sequence may begin anywhere)
        q = torch.full((n + pad, 8, 128), float("nan"), dtype=a["q"].dtype, device=DEV)
        q[at:at + n] = a["q"]
        out, work = torch.full_like(q, 3.0), torch.full((1 << 26,), 255, dtype=torch.uint8, device=DEV)
        B.page_attention(**dict(a, q=q, first=a["first"] + at), out=out, workspace=work)
        assert _same_bits(out[at:at + n], want), (pad, at)
        assert bool((out[:at] == 3).all()) and bool((out[at + n:] == 3).all())


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("hq,most,groups,plens", [(8, 1, (0, 40), [500]), (8, 3, (0, 13, 37), [500, 70]), (4, 2, (3, 4, 20, 40), [90, 16, 333]), (16, 4, (0, 40), [300]), (64, 1, (0, 20), [200]),
                                                  (8, 8, (0, 40), [400]), (8, 12, (0, 40), [100]), (8, 1, (), ())])
def test_sequences_of_more_tokens_than_are_answered(ty, bound, hq, most, groups, plens):
    """More tokens in the arrays than sequences may have: the first max_tokens of each are answered, the others keep what they hold, and nothing behind the
    workspace that was asked for is written."""
    import ctypes as C
    from paper_2604_26334_amd import binding as B
    torch = _t()
    toks = [(5, 1, 17, 0, 2, 9, 3)[i % 7] for i in range(40)]
    lens = [t + i * 5 for i, t in enumerate(toks)]
    a, first, full = T._attend_case(ty, 64, hq, 2, 16, toks, lens, groups, plens, most, bound=bound)
    want = B.page_attention(**a)
    T._check_attend(a, want, first, full, toks, lens, groups, plens, ty)
    p = len(plens)
    sizes = B.ps_page_attention_args(type=0 if ty == "f16" else 1, n_seq=40, n_tokens=sum(toks), n_q_heads=hq, n_kv_heads=2, head_dim=64, page=16, n_pages=a["k_pages"].shape[0],
                                     width=a["table"].shape[1], n_prefix=p, prefix_width=a["prefix_table"].shape[1] if p else 0, max_length=a["max_length"], max_prefix=a.get("max_prefix", 0),
                                     max_tokens=most, scale=0.125)
    need = C.c_uint64()
    assert B.lib().ps_page_attention_workspace(C.byref(sizes), C.byref(need)) == 0
    work = torch.full((need.value + (1 << 24),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full_like(want, 3.0)
    B.page_attention(**dict(a, max_tokens=most), out=out, workspace=work)
    assert bool((work[need.value:] == 255).all())
    for s, t in enumerate(toks):
        kept = slice(first[s] + min(t, most), first[s + 1])
        assert bool((out[kept] == 3).all()), s
        out[kept] = want[kept]
    T._check_attend(a, out, first, full, toks, lens, groups, plens, ty)


@pytest.mark.parametrize("back", [24.0, 24.3, 25.0, 26.5])
def test_weights_far_behind_the_largest(back):
    """One entry at 0 (its weight is exact) and 2^22 - 1 alike `back` nats behind, weights of which may be off by 2^-22 e^-24: top-p keeps the first r with
    1 + (r - 1) w >= p (1 + N w), that is p N - (1 - p) / w behind the first; and an entry is drawn where its share lies."""
    from paper_2604_26334_amd import binding as B
    torch, V = _t(), 1 << 22
    x = torch.full((1, V), -back, device=DEV)
    x[0, 12345] = 0.0
    N, w, e = V - 1, float(np.exp(-float(np.float32(back)))), 2.0 ** -22 * float(np.exp(-24.0))
    for part in (0.25, 0.5, 0.9):
        p = float(np.float32(1 - part * N * w))
        token, kept = B.sample(x, torch.zeros(1, device=DEV), top_p=torch.tensor([p], device=DEV))
        lo, hi = (1 + np.ceil(p * N - (1 - p) / (w + d)) for d in (-e, e))
        assert int(token) == 12345 and lo - 1 <= int(kept) <= hi + 1, (part, lo, int(kept), hi)
    u = float(np.float32(1 - 0.5 * N * w))
    token, kept = B.sample(x, torch.tensor([u], device=DEV))
    lo, hi = (u * N - (1 - u) / (w + d) for d in (-e, e))          # entries of the far ones in front of the drawn one
    assert int(kept) == V and lo - 2 <= int(token) <= hi + 2, (lo, int(token), hi)


@pytest.mark.parametrize("V", [300, 50000])
@pytest.mark.parametrize("temp,size", [(1e-35, 1e-34), (1e-40, 1e-39), (1e-30, 1e-30), (2e-29, 1e-28), (1e-45, 1.0), (1e26, 2e27), (2e27, 1e28), (1e35, 2e35), (3.4e38, 8e37), (float("inf"), 8e37),
                                    (float("inf"), 1.0)])
def test_sample_at_temperatures_of_any_size(temp, size, V):
    """Temperatures and logits at the ends of fp32's range, subnormal ones among them, some logits at the ends of it themselves."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    x = (torch.randn(6, V, generator=_gen(V), device=DEV) * size).clamp(-3.4e38, 3.4e38)
    if size > 1e30:
        x[1, 7], x[2, 9], x[2, 11] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min, float("inf")
    x[3, 5:60] = float("-inf")
    u = torch.rand(6, generator=_gen(1), device=DEV)
    t = torch.full((6,), temp, device=DEV)
    assert float(t[0]) > 0
    for s in (dict(), dict(top_k=_ints([20, 1, 0, 100, V, 3])), dict(top_p=torch.tensor([0.9, 0.5, 0.99, 0.9, 0.1, 0.7], device=DEV)),
              dict(top_k=_ints([200] * 6), top_p=torch.full((6,), 0.8, device=DEV), min_p=torch.full((6,), 0.02, device=DEV))):
        token, kept = B.sample(x, u, temperature=t, **s)
        T._check_sample(x, u, token, kept, temperature=t, **s)


@pytest.mark.parametrize("seed", range(4))
def test_a_steps_attention_sees_what_its_tables_and_rows_say(seed):
    """Tables, rows to pages and attention of one step, the latter against the oracle over the pages as the step left them and the queries as it made
    them: within the roundings of the attention alone, so that a position too many or too few shows."""
    from paper_2604_26334_amd import binding as B
    a = T._step_case(10 + seed)
    pool0, table0, toks = a["pool"].clone(), a["table"].tolist(), a["new"].tolist()
    first, length, position, slot, taken, q, k, out, logits, token, kept = T._step(a, B)
    want = O.page_tables(a["cached"].tolist(), toks, table0, a["free"].tolist(), 1, 16, a["pages"], a["n"], a["offset"].tolist())
    assert a["table"].tolist() == want[0] and slot.tolist()[:len(want[4])] == want[4]
    # the rows of the step's tokens, bit for bit, and no others
    for t, at in enumerate(want[4]):
        pool0[at // 16, 0, :, at % 16], pool0[at // 16, 1, :, at % 16] = k[t], a["v"][t]
    assert _same_bits(a["pool"], pool0)
    seen = dict(q=q, k_pages=a["pool"][:, 0], v_pages=a["pool"][:, 1])
    full = [want[0], a["prefix_table"].tolist()]
    T._check_attend(seen, out, want[1], full, toks, want[2], (0, 4), [50], "f16")
    for lens, plens in (([n - 1 for n in want[2]], [50]), ([n + 1 for n in want[2]], [50]), (want[2], [49])):       # (the check can tell)
        with pytest.raises(AssertionError):
            T._check_attend(seen, out, want[1], full, toks, lens, (0, 4), plens, "f16")


@pytest.mark.parametrize("bound", [0, 1000, 200000])
@pytest.mark.parametrize("most", [2, 40])
def test_a_captured_step_with_room_for_other_batches(bound, most):
    """One captured call in arrays with room for more rows, replayed for several batches: each replay gives what an eager call gives, and leaves the rows behind the
    last sequence alone."""
    from paper_2604_26334_amd import binding as B
    torch = _t()
    room = 12 * most + 500
    batches = []
    for seed in range(3):
        rng = np.random.default_rng(seed)
        toks = [int(rng.integers(0, most + 1)) for _ in range(12)]
        lens = [t + int(rng.integers(0, 300)) for t in toks]
        a, first, full = T._attend_case("f16", 128, 8, 2, 16, toks, lens, (0, 5, 9), [300, 77], seed, bound=bound)
        batches.append((a, first, full, toks, lens))
    q = torch.zeros(room, 8, 128, dtype=torch.float16, device=DEV)
    pages = max(a["k_pages"].shape[0] for a, *_ in batches)
    kp, vp = (torch.zeros(pages, 2, 16, 128, dtype=torch.float16, device=DEV) for _ in range(2))
    width, wide = (max(a[n].shape[1] for a, *_ in batches) for n in ("table", "prefix_table"))
    now = dict(q=q, k_pages=kp, v_pages=vp, first=_ints([0] * 13), length=_ints([0] * 12), table=_ints([[-1] * width] * 12), max_length=max(max(b[4]) for b in batches), max_tokens=most,
               group_first=_ints([0, 5, 9]), prefix_length=_ints([300, 77]), prefix_table=_ints([[-1] * wide] * 2), max_prefix=max(300, bound))

    def put(a):
        n = int(a["first"][-1])
        q.fill_(float("nan"))
        q[:n] = a["q"]
        for name in ("k_pages", "v_pages"):
            now[name][:a[name].shape[0]] = a[name]
        now["first"].copy_(a["first"])
        now["length"].copy_(a["length"])
        now["table"][:, :a["table"].shape[1]] = a["table"]
        now["prefix_table"][:, :a["prefix_table"].shape[1]] = a["prefix_table"]
        return n
    out = torch.full_like(q, 3.0)
    put(batches[0][0])
    B.page_attention(**now, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.page_attention(**now, out=out)
    for i in (0, 1, 2, 0, 2, 1):
        a, first, full, toks, lens = batches[i]
        n = put(a)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert bool((out[n:] == 3).all())
        T._check_attend(a, out[:n], first, full, toks, lens, (0, 5, 9), [300, 77], "f16")
        assert _same_bits(out[:n], B.page_attention(**now)[:n])
