"""Positions, trees and kept paths of one stack that switches between tiers, its caches moving between the arena and the host."""
import numpy as np
import pytest

import synth_inputs as S
from tests import harness as Hn
from tests import test_gpu_draft_step as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tight", [False, True])
def test_a_tree_step_between_prefill_and_decode(tight):
    """A prompt in the 64-token tier, a tree in the 16-token tier whose path is kept, decode in the one-token tier; beside it a stack that decodes
    the same tokens one by one.  Every switch drops the tree and the step to be verified or kept.  Tolerance as between trees and decode token by
    token: fp16 rows on both sides move a score of up to 11 by 2 x 11 x 2^-11, a weight by 1 %, a row by less than twice that."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg = T._cfg(n_layers=2, cap=400)
    W, prompt, n = Hn.WeightCache(cfg, 71), 90, 9
    parents, line = [-1, 0, 0, 1, 1, 2, 3, 5, 6], [0, 1, 3, 6, 8]
    xp, x, xd = (S.activations(71, i, k, cfg["hidden"]) for i, k in ((0, prompt), (1, n), (2, 1)))
    s64 = B.Plan(cfg, 1 << 40, 64).summary()
    budget = s64.workspace_bytes + s64.weight_bytes // 3 if tight else 1 << 28
    table = B.TierTable(cfg, budget)
    tiers = {e.tier_tokens: e.tier for e in table.entries() if e.feasible}
    st, one = B.Stack(table), B.Stack(B.Plan(cfg, 1 << 28, 1))
    for s in (st, one):
        for layer in range(2):
            for kind, expert, N, K in S.matrix_shapes(cfg):
                s.load_matrix(layer, kind, expert, *W(layer, kind, expert))
        s.set_rotation(T._inv_freq(s.device), norm=True)
        s.set_context(0)
    homes = set()

    def tier(tokens):
        st.set_tier(tiers[tokens])
        homes.add(tuple(s.resident for s in st.plan.shards() if s.kind == B.PS_SHARD_KV))
    tier(64)
    xin, xout = T._tensors(st, xp)
    torch.cuda.synchronize()
    B.chunked_forward(st, xin, xout)
    st.synchronize()
    for i in range(prompt):
        one.set_context(i)
        last = T._forward(one, xp[i:i + 1])
    assert Hn.rel_err(xout[-1:].cpu().numpy(), last.cpu().numpy()) <= 2e-2
    tier(16)
    path, count = torch.tensor(line + [-1] * 4, dtype=torch.int32, device=st.device), torch.tensor([5], dtype=torch.int32, device=st.device)
    st.set_tree(parents)
    st.set_context(prompt)
    got = T._forward(st, x).cpu().numpy()
    st.keep_path(path, count)
    for i, node in enumerate(line):
        one.set_context(prompt + i)
        assert Hn.rel_err(got[node:node + 1], T._forward(one, x[node:node + 1]).cpu().numpy()) <= 2e-2, node
    tier(1)
    with pytest.raises(B.PshardError) as e:
        st.keep_path(path[:1].contiguous(), count)
    assert e.value.code == B.PS_E_STATE
    for s in (st, one):
        s.set_context(prompt + len(line))
    assert Hn.rel_err(T._forward(st, xd).cpu().numpy(), T._forward(one, xd).cpu().numpy()) <= 2e-2
    tier(16)                                                            # no tree is set: a chunk of 16
    st.set_context(prompt)
    xin, xout = T._tensors(st, S.activations(71, 3, 16, cfg["hidden"]))
    torch.cuda.synchronize()
    st.forward(xin, xout)
    st.synchronize()
    assert bool(torch.isfinite(xout).all())
    assert len(homes) > 1 or not tight, homes
    st.close()
    one.close()
