"""Attention weights at the ends of their range."""
import numpy as np
import pytest

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
