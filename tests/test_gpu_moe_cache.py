"""An MoE stack whose caches cross PCIe: every step's copies come behind the rows that the step before it appended."""
import numpy as np
import pytest

import synth_inputs as S
from tests import harness as Hn
from tests import test_gpu_draft_step as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers,tokens", [(1, 1), (1, 4), (2, 1)])
def test_streamed_caches_of_an_moe_stack_follow_their_steps(layers, tokens):
    """Twelve steps one behind the other without a wait between them, caches streamed and pinned: the same bits."""
    import torch
    from paper_2604_26334_amd import binding as B
    steps, ctx, cap = 12, 40, 2000
    cfg = T._cfg(n_layers=layers, cap=cap, n_q=4, n_kv=2, moe=True)
    W, caches = Hn.WeightCache(cfg, 61), T._caches(cfg, 61, ctx)
    fs = B.Plan(cfg, 1 << 40, tokens).summary()
    tight = fs.workspace_bytes + 2 * B.Plan(cfg, fs.workspace_bytes + fs.weight_bytes - 4096, tokens).summary().slot_bytes + 4096
    got = []
    for budget in (1 << 30, tight):
        st = T._stack(cfg, W, tokens, ctx, caches, budget)
        kv = [s for s in st.plan.shards() if s.kind == B.PS_SHARD_KV]
        assert any(not s.resident for s in kv) == (budget == tight)
        xs = [torch.from_numpy(S.activations(61, i, tokens, cfg["hidden"])).to(st.device) for i in range(steps)]
        outs = [torch.zeros_like(x) for x in xs]
        torch.cuda.synchronize()
        for i in range(steps):
            st.set_context(ctx + i * tokens)
            st.forward(xs[i], outs[i], S.router_logits(61, i, layers, tokens, cfg["n_experts"]))
        st.synchronize()
        got.append([o.cpu().numpy() for o in outs])
        st.close()
    for a, b in zip(*got):
        assert np.array_equal(a.view(np.uint16), b.view(np.uint16))
