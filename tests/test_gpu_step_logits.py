"""Which logits a stack's forward writes and which a verification judges: rows that lie in the forward, buffers that are large enough,
and what the last forward did rather than what is set for the next."""
import ctypes as C

import numpy as np
import pytest

import synth_inputs as S
from oracle import drafts as D
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


def _draft(st, n, seed):
    import torch
    rng = np.random.default_rng(seed)
    token = rng.integers(0, V, size=n)
    return (torch.tensor(token, dtype=torch.int32, device=st.device), torch.tensor(rng.random(n) * 0.2, dtype=torch.float32, device=st.device),
            torch.tensor(rng.random(1), dtype=torch.float32, device=st.device))


def _check(got, logits, token, parents, u, us):
    path, count, nxt = (t.cpu().tolist() for t in got)
    want, w_next = D.verify_tree(logits.double().cpu().numpy(), token.tolist(), parents, u.tolist(), float(us[0]))
    assert path == want + [-1] * (len(parents) - len(want)) and count == [len(want)] and nxt == [w_next]


def test_verification_needs_a_forward_that_wrote_logits():
    import torch
    from paper_2604_26334_amd import binding as B
    cfg, st, _ = _head_stack()
    n = len(PARENTS)
    st.set_tree(PARENTS)
    x = S.activations(52, 0, n, cfg["hidden"])
    token, u, us = _draft(st, n, 1)
    T._forward(st, x)                                                       # the head was off
    logits = torch.zeros(PLAN, V, dtype=torch.float16, device=st.device)
    st.set_logits_out(logits, 0, PLAN)
    _refused(B.PS_E_STATE, st.verify_tree, token, u, us)
    one = torch.zeros(V, dtype=torch.float16, device=st.device)
    st.set_logits_out(one, 0, 1)
    _refused(B.PS_E_STATE, st.verify_tree, token[:1].contiguous(), u[:1].contiguous(), us)
    a = B.ps_stack_verify_args(*[1 << 30] * 8, 2, 0)
    need = C.c_uint64()
    assert B.lib().ps_stack_verify_workspace(st.h, C.byref(a), C.byref(need)) == B.PS_E_STATE
    # a prompt in chunks is no tree's step, whatever it wrote
    st.set_tree()
    st.set_logits_out(logits, 0, PLAN)
    T._forward(st, S.activations(52, 1, PLAN, cfg["hidden"]))
    st.set_context(CTX)
    xin, xout = T._tensors(st, S.activations(52, 2, 11, cfg["hidden"]))
    B.chunked_forward(st, xin, xout)
    st.synchronize()
    token, u, us = _draft(st, PLAN, 2)
    _refused(B.PS_E_STATE, st.verify_tree, token, u, us)
    st.close()


@pytest.mark.parametrize("then", ["other buffer", "one token", "off"])
def test_verification_judges_what_the_last_forward_wrote(then):
    """The next step's logits may be set before this one's are judged."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg, st, _ = _head_stack()
    n = len(PARENTS)
    st.set_tree(PARENTS)
    x = S.activations(53, 0, n, cfg["hidden"])
    token, u, us = _draft(st, n, 3)
    logits = torch.zeros(PLAN, V, dtype=torch.float16, device=st.device)
    st.set_logits_out(logits, 0, PLAN)
    T._forward(st, x)
    token[1] = int(logits[0].float().argmax())
    other = torch.zeros(PLAN, V, dtype=torch.float16, device=st.device)
    other[:, 3] = 60.0                                                      # where it is judged instead, token 3 follows everything
    torch.cuda.synchronize()
    if then == "other buffer":
        st.set_logits_out(other, 0, PLAN)
    elif then == "one token":
        st.set_logits_out(other[0].contiguous(), 2, 1)
    else:
        st.set_logits_out(None, 0, 0)
    us.fill_(0.0)                                                           # the first token that has any weight: 0 in these logits
    torch.cuda.synchronize()
    got = st.verify_tree(token, u, us)
    st.synchronize()
    _check(got, logits[:n], token, PARENTS, u, us)
    _refused(B.PS_E_ARG, st.verify_tree, token[:1].contiguous(), u[:1].contiguous(), us)      # one number per row of that forward
    st.keep_path(got[0], got[1])
    st.close()


def test_one_tokens_logits_are_judged_alone_whatever_is_set_next():
    import torch
    from paper_2604_26334_amd import binding as B
    cfg, st, _ = _head_stack()
    x = S.activations(54, 0, PLAN, cfg["hidden"])
    one = torch.zeros(V, dtype=torch.float16, device=st.device)
    st.set_logits_out(one, 4, 1)
    T._forward(st, x)
    rows = torch.zeros(PLAN, V, dtype=torch.float16, device=st.device)
    st.set_logits_out(rows, 0, PLAN)
    token, u, us = _draft(st, PLAN, 4)
    torch.cuda.synchronize()
    _refused(B.PS_E_ARG, st.verify_tree, token, u, us)
    t1, u1 = token[:1].contiguous(), u[:1].contiguous()
    torch.cuda.synchronize()
    got = st.verify_tree(t1, u1, us)
    st.synchronize()
    _check(got, one[None], t1, [-1], u1, us)
    st.close()


def test_logits_set_in_one_tier_fit_the_forwards_of_another():
    """A buffer set for fewer rows than the new tier's forward has, or a token that it does not have, is refused before anything is enqueued."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg = dict(Hn.small_dense_cfg(1), vocab=V)
    W, head = Hn.WeightCache(cfg, 55), S.head_matrix(55, cfg)
    table = B.TierTable(cfg, 1 << 28)
    tiers = {e.tier_tokens: e.tier for e in table.entries() if e.feasible}
    st = B.Stack(table)
    for kind, expert, N, K in S.matrix_shapes(cfg):
        st.load_matrix(0, kind, expert, *W(0, kind, expert))
    st.load_matrix(1, S.MAT_OUT, None, *head)
    few, many = 16, 64
    x = {n: S.activations(55, n, n, cfg["hidden"]) for n in (1, few, many)}
    buf = torch.full((many + 1, V), 7.0, dtype=torch.float16, device=st.device)

    def refused(n):
        xin, xout = T._tensors(st, x[n])
        torch.cuda.synchronize()
        for call in (st.forward, st.forward_noalloc):
            _refused(B.PS_E_STATE, call, xin, xout)
        st.synchronize()
        assert bool((xout == 0).all()) and bool((buf == 7).all())

    def right(n, rows):
        out = T._forward(st, x[n]).cpu().numpy()
        got = buf[:len(rows)].cpu().numpy()
        assert Hn.rel_err(got, O.output_head(out[rows], cfg, head, mirror=True)) <= 5e-3
        assert bool((buf[len(rows):] == 7).all())
        buf.fill_(7.0)
        torch.cuda.synchronize()
    st.set_tier(tiers[few])
    st.set_logits_out(buf[:few], 0, few)
    st.set_tier(tiers[many])
    refused(many)
    st.set_tier(tiers[few])
    right(few, list(range(few)))
    st.set_logits_out(buf[0], few - 1, 1)
    st.set_tier(tiers[1])
    refused(1)
    st.set_tier(tiers[many])
    right(many, [few - 1])
    st.set_logits_out(buf[:many], 0, many)
    st.set_tier(tiers[few])                       # (a larger buffer than the forward needs)
    right(few, list(range(few)))
    st.close()
