"""Weights of the attention over pages at the ends of their range."""
import numpy as np
import pytest

from oracle import batch as O
from tests import test_gpu_batch as T
from tests.test_gpu_drafts import DEV, _dt, _gen, _half_step, _ints, _np

pytestmark = pytest.mark.gpu


def _paged(k, v, page, heads):
    """Rows [positions, d] as pages of one head that stands for all: pages [n, heads, page, d] and their numbers"""
    import torch
    n = -(-k.shape[0] // page)
    pages = torch.zeros(2, n, 1, page, k.shape[1], dtype=k.dtype, device=DEV)
    for x, p in ((k, pages[0]), (v, pages[1])):
        p.view(n * page, -1)[:x.shape[0]] = x
    return pages[0].expand(n, heads, page, k.shape[1]), pages[1].expand(n, heads, page, k.shape[1]), list(range(n))


def _call(q, k, v, prefix, scale, bound=0):
    """t tokens of one sequence over `prefix` positions of a prefix and the others of its own, the tokens' own positions last; bound: of the prefix
    (a long one is dealt with by itself)"""
    import torch
    from paper_2604_26334_amd import binding as B
    t, heads, page = q.shape[0], q.shape[1], 16
    own = k.shape[0] - prefix
    cut = -(-prefix // page) * page
    pad = torch.full((cut - prefix, k.shape[1]), float("nan"), dtype=k.dtype, device=DEV)
    kp, vp, numbers = _paged(torch.cat((k[:prefix], pad, k[prefix:])), torch.cat((v[:prefix], pad, v[prefix:])), page, heads)
    pre = dict(group_first=_ints([0, 1]), prefix_length=_ints([prefix]), prefix_table=_ints([numbers[:cut // page] + [-1] * (bound // page)]), max_prefix=max(prefix, bound)) if prefix else {}
    return B.page_attention(q, kp, vp, _ints([0, t]), _ints([own]), _ints([numbers[cut // page:]]), max_length=own, max_tokens=t, scale=scale, **pre)


@pytest.mark.parametrize("bound", [0, 200000])
@pytest.mark.parametrize("ty,size", [("f16", 10240.0), ("bf16", 2.0 ** 24)])
@pytest.mark.parametrize("d,hq,toks,lens,groups,plens", [(128, 4, [1, 2], [300, 40], (0, 2), [700]), (64, 8, [3, 1], [1000, 40], (), ()),
                                                         (128, 4, [1] * 40, [50] * 40, (0, 40), [600]), (64, 4, [50, 20], [90, 300], (0, 2), [200])])
def test_scores_of_any_size(ty, size, d, hq, toks, lens, groups, plens, bound):
    """Queries and keys so large that one position's weight is 1 and all others are 0: that position's value, bit for bit.  Rows whose two
    largest scores lie closer than that (a product of 200 sqrt(d) is 200 nats) or than the fp32 sum of d products may be off (2 d 2^-24 of the sum of
    their sizes) are left out."""
    from paper_2604_26334_amd import binding as B
    a, first, full = T._attend_case(ty, d, hq, 2, 16, toks, lens, groups, plens, 5, bound=bound)
    a["q"], a["k_pages"] = a["q"] * size, a["k_pages"] * size
    out, q, kp, vp = (_np(x) for x in (B.page_attention(**a), a["q"], a["k_pages"], a["v_pages"]))
    seen = left = 0
    for s, (t, length) in enumerate(zip(toks, lens)):
        k, v = (O.rows_of(x, full[0][s], length)[0] for x in (kp, vp))
        p = 0
        for i, pl in enumerate(plens):
            if groups[i] <= s < groups[i + 1]:
                p, k, v = pl, np.concatenate([O.rows_of(kp, full[1][i], pl)[0], k], 1), np.concatenate([O.rows_of(vp, full[1][i], pl)[0], v], 1)
        for i in range(t):
            n = p + length - t + i + 1
            for h in range(hq):
                kk, vv, x = k[h // (hq // 2), :n], v[h // (hq // 2), :n], q[first[s] + i, h]
                z = kk @ x
                best = np.argsort(z)[-2:]
                seen += 1
                if z[best[1]] - z[best[0]] <= 2 * d * 2.0 ** -24 * (np.abs(kk[best]) @ np.abs(x)).max() + 200 * d ** 0.5:
                    left += 1
                    continue
                assert np.array_equal(out[first[s] + i, h], vv[best[1]]), (s, i, h)
    assert left * 10 <= seen


@pytest.mark.parametrize("bound", [0, 200000])
@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("d,t,prefix", [(64, 1, 0), (128, 2, 0), (128, 2, 2000), (64, 40, 0), (128, 40, 3000), (64, 1, 3900)])
@pytest.mark.parametrize("spot", [0, 2005, 3995])
def test_small_weights_add_up(ty, d, t, prefix, spot, bound):
    """One key `gap` nats ahead, whose value is zero, and 4000 alike with values about 100: what comes out is these alone.  The tolerance: a half
    step of the result, half a step of every weight and of their sum, weights held to 2^-35 of the largest where the type's half step ends (half of
    fp16's least step 2^-24 under a largest weight of 2^10 or more), scores and their exponentials in fp32 (a score of up to 20, 29 in powers of two:
    2^-19 of a weight; 2^-17 allowed)."""
    import torch
    heads, n, dt, scale = 8, 4000, _dt(ty), 2.0 ** -3
    g = _gen(7)
    for gap in (10.0, 14.0, 18.0, 20.0):
        q = torch.zeros(t, heads, d, dtype=dt, device=DEV)
        q[..., 0] = 16.0
        k = torch.zeros(n + t, d, dtype=dt, device=DEV)
        v = (100 + 10 * torch.rand(n + t, d, generator=g, device=DEV)).to(dt)
        k[spot, 0] = gap / 2
        v[spot] = 0
        out = _call(q, k, v, prefix, scale, bound)
        ref = O.attention(_np(q[:, :1]), _np(k)[None], _np(v)[None], np.ones(n + t, bool), n, scale)
        least = 2.0 ** -35 if ty == "f16" else 2.0 ** -100
        tol = np.abs(ref) * (3 * _half_step(ty) + 2.0 ** -17) + 2 * n * least * 110
        off = np.abs(_np(out) - ref) / tol
        assert off.max() <= 1, (gap, off.max())


@pytest.mark.parametrize("bound", [0, 200000])
@pytest.mark.parametrize("t,prefix", [(2, 0), (2, 500), (40, 0), (40, 500)])
def test_large_values_do_not_overflow(t, prefix, bound):
    """bf16 values of 2^117 to 2^118 behind keys that rise by 5.2 nats after the first 128: 900 weights of at most 1 times these add up to less
    than 2^128, within fp32.  All values alike in a dimension: the result is that value, to the rounding of the result (half a step) and of a weight
    sum against the weighted sum, both of the same rounded weights in fp32 (900 x 2^-24 each)."""
    import torch
    n, d, dt = 900, 128, torch.bfloat16
    q = torch.zeros(t, 8, d, dtype=dt, device=DEV)
    q[..., 0] = 16.0
    row = ((1 + torch.rand(d, generator=_gen(3), device=DEV)) * 2.0 ** 117).to(dt)
    k = torch.zeros(n, d, dtype=dt, device=DEV)
    k[128:, 0] = 2.6
    out = _call(q, k, row.expand(n, d), prefix, 2.0 ** -3, bound)
    ref = _np(row)
    assert (np.abs(_np(out) - ref) <= ref * (2.0 ** -8 + 900 * 2.0 ** -23)).all()
