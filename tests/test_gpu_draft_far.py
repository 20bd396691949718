"""Operators of drafted tokens where offsets pass 32 bits, and at the largest vocabulary."""
import numpy as np
import pytest

from tests import test_gpu_drafts as T

pytestmark = pytest.mark.gpu


def test_rope_of_rows_far_apart():
    """Tokens 2^24 elements apart, 300 of them: 5 x 10^9 elements; the same bits as rows together."""
    import torch
    from paper_2604_26334_amd import binding as B
    n, step = 300, 1 << 24
    buf = torch.empty(n * step, dtype=torch.float16, device=T.DEV)
    for d in (128, 40):
        far = buf.as_strided((n, 2, d), (step, d, 1))
        near = torch.randn(n, 2, d, generator=T._gen(1), device=T.DEV).half()
        far.copy_(near)
        pos, inv = T._ints(list(range(n))), torch.full((d // 2,), 0.01, device=T.DEV)
        want, _ = B.qk_norm_rope(near, near[:, :0], pos, inv)
        got, _ = B.qk_norm_rope(far, near[:, :0], pos, inv, q_out=far, k_out=near[:, :0])
        assert T._same_bits(got, want)


@pytest.mark.parametrize("drafts", [True, False])
def test_verification_of_rows_far_apart(drafts):
    """Rows 2^24 entries apart, sequences behind element 2^32."""
    import torch
    from paper_2604_26334_amd import binding as B
    rng = np.random.default_rng(2)
    a, first = T._verify_case("f16", rng, [5, 3], 5000, "tree", drafts, [0.9, 1.0])
    want = B.verify_tree(**a, max_tree=5, max_children=3)
    T._check_verify(a, want, first, [5, 3], 5, 3)
    lead, step = 290, 1 << 24
    n = lead + 8
    for name in ("target_logits", "draft_logits"):
        if a[name] is not None:
            rows = torch.empty(n * step, dtype=torch.float16, device=T.DEV).as_strided((n, 5000), (step, 1))
            rows[lead:] = a[name]
            a[name] = rows
    for name in ("token", "parent", "u_accept"):
        a[name] = torch.cat((torch.zeros(lead, dtype=a[name].dtype, device=T.DEV), a[name]))
    a["first"] = T._ints([lead, lead + 5, lead + 8])
    got = B.verify_tree(**a, max_tree=5, max_children=3)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("drafts", [True, False])
def test_verification_of_the_largest_vocabulary(drafts):
    import torch
    from paper_2604_26334_amd import binding as B
    V, trees = 1 << 24, [3, 1]
    rng = np.random.default_rng(3)
    target = torch.randn(4, V, generator=T._gen(5), device=T.DEV) * 3
    draft = target * 0.9 + torch.randn(4, V, generator=T._gen(6), device=T.DEV)
    token = [0, int(draft[0].argmax()), int(draft[0].topk(2).indices[1]), 7]
    for us in (0.0, 0.5, 1 - 2.0 ** -24):
        a = dict(target_logits=target, draft_logits=draft if drafts else None, token=T._ints(token), parent=T._ints([-1, 0, 0, -1]), first=T._ints([0, 3, 4]),
                 u_accept=torch.tensor(rng.random(4), dtype=torch.float32, device=T.DEV), u_sample=torch.tensor([us, us], dtype=torch.float32, device=T.DEV),
                 temperature=torch.tensor([0.7, 1.0], device=T.DEV))
        T._check_verify(a, B.verify_tree(**a, max_tree=3, max_children=2), [0, 3, 4], trees, 3, 2)


def test_kept_rows_far_apart():
    """Planes and sequences more than 2^32 bytes apart."""
    import torch
    from paper_2604_26334_amd import binding as B
    plane, seq, cap, d = 1 << 29, 5 << 29, 40, 64
    buf = torch.empty(2 * seq, dtype=torch.float16, device=T.DEV)
    far = buf.as_strided((2, 5, cap, d), (seq, plane, d, 1))
    near = torch.randn(2, 5, cap, d, generator=T._gen(2), device=T.DEV).half()
    far.copy_(near)
    path, count, ctx = T._ints([[0, 2, 5, -1, -1, -1], [0, 1, 3, 4, -1, -1]]), T._ints([3, 4]), T._ints([30, 3])
    want = B.cache_keep(near, path, count, ctx)
    assert T._same_bits(B.cache_keep(far, path, count, ctx), want)
