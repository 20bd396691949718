"""A sequence's verification alone, in a batch, and under a larger bound on the trees' size, against the oracle."""
import numpy as np
import pytest

from tests import test_gpu_drafts as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty,vocab", [("f16", 32003), ("f32", 9001), ("bf16", 50257)])
@pytest.mark.parametrize("drafts", [True, False])
def test_a_sequence_alone_and_among_others(ty, vocab, drafts):
    from paper_2604_26334_amd import binding as B
    rng = np.random.default_rng(vocab + drafts)
    trees = [(7, 1, 12, 4)[i % 4] for i in range(32)]
    temps = [(0.8, 1.0, 1.4)[i % 3] for i in range(32)]
    a, first = T._verify_case(ty, rng, trees, vocab, "tree", drafts, temps, spread=2.5)
    T._check_verify(a, B.verify_tree(**a, max_tree=12, max_children=4), first, trees, 12, 4)
    T._check_verify(a, B.verify_tree(**a, max_tree=256, max_children=4), first, trees, 256, 4)
    rows = ("target_logits", "draft_logits", "token", "parent", "u_accept")
    for s in (0, 2, 5, 30):
        r = slice(first[s], first[s + 1])
        b = {n: None if a[n] is None else a[n][r] for n in rows}
        b.update(first=T._ints([0, trees[s]]), u_sample=a["u_sample"][s:s + 1], temperature=a["temperature"][s:s + 1])
        for bound in (trees[s], 12, 256):
            T._check_verify(b, B.verify_tree(**b, max_tree=bound, max_children=4), [0, trees[s]], [trees[s]], bound, 4)
