"""Which logits a stack's forward writes: of rows that lie in it."""
import pytest

import synth_inputs as S
from oracle import oracle as O
from tests import harness as Hn
from tests import test_gpu_draft_step as T

pytestmark = pytest.mark.gpu

V, CTX, PLAN = 400, 20, 8
PARENTS = [-1, 0, 0, 1, 2]


def _head_stack(seed=51, cap=80):
    cfg = T._cfg(n_layers=1, cap=cap, vocab=V)
    W, caches, head = Hn.WeightCache(cfg, seed), T._caches(cfg, seed, CTX), S.head_matrix(seed, cfg)
    return cfg, T._stack(cfg, W, PLAN, CTX, caches, head=head), head


def _refused(code, call, *args, **kw):
    from paper_2604_26334_amd import binding as B
    with pytest.raises(B.PshardError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_one_tokens_logits_are_of_a_row_of_the_tree():
    """The token whose logits are asked for has to be a row of the forward: a tree may have fewer than the plan."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg, st, head = _head_stack()
    n = len(PARENTS)
    x = S.activations(51, 0, n, cfg["hidden"])
    one = torch.full((V,), 7.0, dtype=torch.float16, device=st.device)
    xin, xout = T._tensors(st, x)
    st.set_tree(PARENTS)
    for first in (n, PLAN - 1):
        st.set_logits_out(one, first, 1)
        torch.cuda.synchronize()
        _refused(B.PS_E_STATE, st.forward, xin, xout)
        st.synchronize()
        assert bool((xout == 0).all()) and bool((one == 7).all())           # nothing was enqueued
    # the last row of the tree is one, and a chunk has all of the plan's
    st.set_logits_out(one, n - 1, 1)
    out = T._forward(st, x).cpu().numpy()
    assert Hn.rel_err(one.cpu().numpy()[None], O.output_head(out[n - 1:], cfg, head, mirror=True)) <= 5e-3
    st.set_tree()
    st.set_logits_out(one, PLAN - 1, 1)
    out = T._forward(st, S.activations(51, 1, PLAN, cfg["hidden"])).cpu().numpy()
    assert Hn.rel_err(one.cpu().numpy()[None], O.output_head(out[PLAN - 1:], cfg, head, mirror=True)) <= 5e-3
    st.close()

