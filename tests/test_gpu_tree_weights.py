"""Attention weights at the ends of their range."""
import numpy as np
import pytest

from oracle import drafts as D
from tests import test_gpu_drafts as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty,size", [("f16", 10240.0), ("bf16", 2.0 ** 24)])
@pytest.mark.parametrize("d,hq,hk,trees,ctxs", [(128, 4, 2, [5], [300]), (64, 8, 2, [9, 3], [1000, 40]), (128, 4, 1, [40], [700]), (64, 2, 2, [60], [90])])
def test_scores_of_any_size(ty, size, d, hq, hk, trees, ctxs):
    """Queries and keys so large that one position's weight is 1 and all others are 0: that position's value, bit for bit.  Rows whose
    two largest scores lie closer than that (a product of 200 sqrt(d) is 200 nats) or than the fp32 sum of d products may be off (2 d 2^-24 of the sum of
    their sizes) are left out."""
    from paper_2604_26334_amd import binding as B
    cap = max(ctxs) + 64
    a, first, parent = T._attention_case(ty, d, hq, hk, trees, ctxs, cap, "tree", 5)
    for name in ("q", "k_new", "k_cache"):
        a[name] = a[name] * size
    out = T._np(B.tree_attention(**a, max_context=max(ctxs), max_tree=max(trees)))
    q, kn, vn, kc, vc = (T._np(a[n]) for n in ("q", "k_new", "v_new", "k_cache", "v_cache"))
    seen = left = 0
    for s, (t, c) in enumerate(zip(trees, ctxs)):
        for i in range(t):
            line, j = [], i
            while j >= 0:
                line.append(first[s] + j)
                up = parent[first[s] + j]
                j = up if 0 <= up < j else -1
            for h in range(hq):
                k = np.concatenate([kc[s, h // (hq // hk), :c], kn[line, h // (hq // hk)]])
                v = np.concatenate([vc[s, h // (hq // hk), :c], vn[line, h // (hq // hk)]])
                x = q[first[s] + i, h]
                z = k @ x
                best = np.argsort(z)[-2:]
                seen += 1
                if z[best[1]] - z[best[0]] <= 2 * d * 2.0 ** -24 * (np.abs(k[best]) @ np.abs(x)).max() + 200 * d ** 0.5:
                    left += 1
                    continue
                assert np.array_equal(out[first[s] + i, h], v[best[1]]), (s, i, h)
    assert left * 10 <= seen


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("d,t", [(64, 1), (128, 2), (64, 20), (128, 40), (64, 40)])
@pytest.mark.parametrize("spot", ["first", "middle", "own"])
def test_small_weights_add_up(ty, d, t, spot):
    """One key `gap` nats ahead, whose value is zero, and 4000 alike with values about 100: what comes out is these alone.  512 heads, so
    that a head's positions are not split.  The tolerance: a half step of the result, half a step of every weight and of
    their sum, weights held to 2^-35 of the largest where the type's half step ends (half of fp16's least step 2^-24 under a largest weight of 2^10 or
    more), scores and their exponentials in fp32 (a score of up to 20, 29 in powers of two: 2^-19 of a weight; 2^-17 allowed)."""
    import torch
    from paper_2604_26334_amd import binding as B
    heads, n, dt = 512, 4000, T._dt(ty)
    g = T._gen(7)
    at = {"first": 0, "middle": n // 2 + 5, "own": None}[spot]
    scale = 2.0 ** -3
    for gap in (10.0, 14.0, 16.0, 18.0, 20.0):
        q = torch.zeros(t, heads, d, dtype=dt, device=T.DEV)
        q[..., 0] = 16.0
        kc = torch.zeros(1, 1, n, d, dtype=dt, device=T.DEV)
        vc = (100 + 10 * torch.rand(1, 1, n, d, generator=g, device=T.DEV)).to(dt)
        kn = torch.zeros(t, 1, d, dtype=dt, device=T.DEV)
        vn = (100 + 10 * torch.rand(t, 1, d, generator=g, device=T.DEV)).to(dt)
        if at is None:
            kn[0, 0, 0] = gap / 2                                     # every node comes behind node 0
            vn[0] = 0
        else:
            kc[0, 0, at, 0] = gap / 2
            vc[0, 0, at] = 0
        parent = [-1] + [0] * (t - 1)
        out = B.tree_attention(q, kn.expand(t, heads, d), vn.expand(t, heads, d), kc.expand(1, heads, n, d), vc.expand(1, heads, n, d),
                               T._ints([0, t]), T._ints([n]), T._ints(parent), max_context=n, max_tree=t, scale=scale)
        ref = D.tree_attention(T._np(q[:, :1]), T._np(kn), T._np(vn), T._np(kc[0]), T._np(vc[0]), n, parent, scale)
        hs = T._half_step(ty)
        least = 2.0 ** -35 if ty == "f16" else 2.0 ** -100
        tol = np.abs(ref) * (3 * hs + 2.0 ** -17) + 2 * n * least * 110
        off = np.abs(T._np(out) - ref) / tol
        assert off.max() <= 1, (gap, off.max())


@pytest.mark.parametrize("t", [2, 20, 40])
def test_large_values_do_not_overflow(t):
    """bf16 values of 2^117 to 2^118 behind keys that rise by 5.2 nats after the first 128: 900 weights of at most 1 times these add up to less
    than 2^128, within fp32 (weights of 2^7.5 would not).  All values alike in a dimension: the result is that value, to the rounding of the result (half a
    step) and of a weight sum against the weighted sum, both of the same rounded weights in fp32 (900 x 2^-24)."""
    import torch
    from paper_2604_26334_amd import binding as B
    heads, n, d, dt = 512, 900, 128, torch.bfloat16
    q = torch.zeros(t, heads, d, dtype=dt, device=T.DEV)
    q[..., 0] = 16.0
    row = ((1 + torch.rand(d, generator=T._gen(3), device=T.DEV)) * 2.0 ** 117).to(dt)
    kc, kn = torch.zeros(1, 1, n, d, dtype=dt, device=T.DEV), torch.zeros(t, 1, d, dtype=dt, device=T.DEV)
    kc[:, :, 128:, 0] = 2.6
    kn[..., 0] = 2.6
    vc, vn = row.expand(1, heads, n, d), row.expand(t, heads, d)
    vc, vn = vc[:, :1].contiguous().expand(1, heads, n, d), vn[:, :1].contiguous().expand(t, heads, d)
    out = B.tree_attention(q, kn.expand(t, heads, d), vn, kc.expand(1, heads, n, d), vc, T._ints([0, t]), T._ints([n]), T._ints([-1] * t),
                           max_context=n, max_tree=t, scale=2.0 ** -3)
    ref = T._np(row)
    assert (np.abs(T._np(out) - ref) <= ref * (2.0 ** -8 + 900 * 2.0 ** -23)).all()
