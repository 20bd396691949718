"""Rotation, trees of drafted tokens, verification and kept paths inside a stack's forwards, against the float64 oracle on the very rows the
stack's projections left, and against the stack's own token-by-token decode."""
import ctypes as C

import numpy as np
import pytest

import synth_inputs as S
from oracle import drafts as D
from tests import harness as Hn

pytestmark = pytest.mark.gpu


def _cfg(n_layers=1, cap=400, n_q=4, n_kv=2, vocab=0, moe=False):
    base = Hn.small_moe_cfg(n_layers) if moe else Hn.small_dense_cfg(n_layers)
    cfg = dict(base, kv_context=cap, n_q_heads=n_q, n_kv_heads=n_kv)
    return dict(cfg, vocab=vocab) if vocab else cfg


def _stack(cfg, W, tokens, ctx, caches, budget=1 << 30, mode=0, head=None):
    from paper_2604_26334_amd import binding as B
    plan = B.Plan(cfg, budget, tokens)
    st = B.Stack(plan)
    st.set_decode_mode(mode)
    for layer in range(cfg["n_layers"]):
        for kind, expert, N, K in S.matrix_shapes(cfg):
            st.load_matrix(layer, kind, expert, *W(layer, kind, expert))
        for g in range(cfg["n_kv_heads"]):
            st.load_kv(layer, g, caches[layer][0][g], caches[layer][1][g])
    if head is not None:
        st.load_matrix(cfg["n_layers"], S.MAT_OUT, None, *head)
    st.set_context(ctx)
    return st


def _caches(cfg, seed, ctx):
    return [S.kv_cache(seed, l, cfg["n_kv_heads"], ctx, 128) for l in range(cfg["n_layers"])]


def _tensors(st, x):
    import torch
    xin = torch.from_numpy(np.ascontiguousarray(x)).to(st.device)
    return xin, torch.zeros_like(xin)


def _forward(st, x, lg=None):
    import torch
    xin, xout = _tensors(st, x)
    torch.cuda.synchronize()
    st.forward(xin, xout, lg)
    st.synchronize()
    return xout


def _inv_freq(dev, rot=128):
    import torch
    return torch.tensor(np.exp(-np.arange(rot // 2) / (rot // 2) * np.log(10000.0)), dtype=torch.float32, device=dev)


def _tree_parents(rng, n):
    return [-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, n)]


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _check_rows(cfg, qkv, attn, K, V, ctx, parents):
    """Attention rows against the oracle on the stored fp16 rows: half a step of the result (2^-11), the weights' rounding (2^-11 of each, and
    of their sum where it is taken of the unrounded ones: 2^-10 of the largest value), scores in fp32 (138 terms' roundings of their size)."""
    n_q, n_kv = cfg["n_q_heads"], cfg["n_kv_heads"]
    q, k, v = (qkv[:, a:b].astype(np.float64) for a, b in ((0, n_q), (n_q, n_q + n_kv), (n_q + n_kv, n_q + 2 * n_kv)))
    Kd, Vd = np.asarray(K, dtype=np.float64), np.asarray(V, dtype=np.float64)
    ref = D.tree_attention(q, k, v, Kd, Vd, ctx, parents, 128 ** -0.5)
    v_max = max(np.abs(v).max(), np.abs(Vd[:, :ctx]).max() if ctx else 0)
    k_max = max(np.abs(k).max(), np.abs(Kd[:, :ctx]).max() if ctx else 0)
    size = np.abs(q).sum(-1).max() * k_max * 128 ** -0.5
    tol = np.abs(ref) * 2.0 ** -11 + 2 * v_max * (2.0 ** -11 + 138 * size * 2.0 ** -24 / 16) + 1e-6
    off = np.abs(attn.astype(np.float64) - ref) / tol
    assert off.max() <= 1, off.max()


@pytest.mark.parametrize("M,mode,ctx,rot,pairs,norm", [(1, 0, 37, 128, False, True), (1, 3, 37, 128, False, True), (1, 3, 0, 64, True, False), (4, 0, 5, 128, False, True),
                                                       (16, 0, 90, 64, True, True), (70, 0, 33, 128, False, False), (300, 0, 20, 0, False, True)])
def test_a_forward_turns_its_queries_and_keys(M, mode, ctx, rot, pairs, norm):
    import torch
    cfg = _cfg(cap=ctx + M + 8)
    W, caches = Hn.WeightCache(cfg, 31), _caches(cfg, 31, ctx)
    st = _stack(cfg, W, M, ctx, caches, mode=mode)
    x = S.activations(31, 0, M, cfg["hidden"])
    rows = cfg["n_q_heads"] + 2 * cfg["n_kv_heads"]
    plain_out = _forward(st, x)
    plain = st.debug_buffer(0, np.float16, (M, rows, 128)).copy()
    rng = np.random.default_rng(5)
    gq, gk = (torch.tensor(1 + 0.2 * rng.normal(size=(1, 128)), dtype=torch.float16, device=st.device) for _ in range(2))
    inv = _inv_freq(st.device, rot) if rot else None
    st.set_rotation(inv, gq if norm else None, gk if norm else None, pairs=pairs, norm=norm)
    for _ in range(2):           # (the second replays a captured step)
        st.set_context(ctx)
        turned_out = _forward(st, x)
        qkv = st.debug_buffer(0, np.float16, (M, rows, 128)).copy()
        attn = st.debug_buffer(5, np.float16, (M, cfg["n_q_heads"], 128)).copy()
        pos = [ctx + i for i in range(M)]
        inv_np = inv.cpu().numpy() if rot else np.zeros(0, np.float32)
        n_q, n_k = cfg["n_q_heads"], cfg["n_q_heads"] + cfg["n_kv_heads"]
        for a, b, g in ((0, n_q, gq), (n_q, n_k, gk)):
            ref = D.qk_norm_rope(plain[:, a:b].astype(np.float64), g.double().cpu().numpy()[0], pos, inv_np, cfg["rms_eps"], norm, pairs)
            # half a step of the value, and fp32 in front of it (152 roundings of the row's largest value allowed)
            tol = np.abs(ref) * 2.0 ** -11 + np.abs(ref).max(-1, keepdims=True) * 152 * 1.5 * 2.0 ** -24 + 1e-7
            assert (np.abs(qkv[:, a:b].astype(np.float64) - ref) <= tol).all()
        assert np.array_equal(qkv[:, n_k:].view(np.uint16), plain[:, n_k:].view(np.uint16))
        _check_rows(cfg, qkv, attn, caches[0][0], caches[0][1], ctx, [i - 1 for i in range(M)])
    if mode == 3:
        assert st.stats().graph_replay == 1
    # and without it again: the former bits
    st.set_rotation()
    st.set_context(ctx)
    again = _forward(st, x)
    same = torch.equal(again, plain_out)
    changed = not torch.equal(again, turned_out)
    assert same and changed == (ctx + M > 1)             # (a token that sees itself alone weighs it 1, however it is turned)
    st.close()


@pytest.mark.parametrize("n_q,n_kv,plan_tokens,n,ctx", [(4, 2, 8, 8, 0), (4, 2, 8, 5, 33), (8, 1, 16, 16, 300), (32, 8, 24, 24, 1000), (4, 4, 64, 61, 200), (2, 2, 300, 256, 40),
                                                       (8, 2, 300, 7, 700), (4, 2, 2, 2, 64), (4, 2, 8, 1, 50)])
def test_a_tree_of_drafts_in_a_forward(n_q, n_kv, plan_tokens, n, ctx):
    """Rows of the tree against the oracle, the same bits with the cache pinned and streamed; the rows appended, then the accepted path's
    put in place, checked in the cache and through the next forward."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg = _cfg(cap=ctx + max(n, plan_tokens) + 30, n_q=n_q, n_kv=n_kv)
    W, caches, rng = Hn.WeightCache(cfg, 33), _caches(cfg, 33, ctx), np.random.default_rng(n)
    parents, rows = _tree_parents(rng, n), n_q + 2 * n_kv
    x, x2 = S.activations(33, 0, n, cfg["hidden"]), S.activations(33, 1, n, cfg["hidden"])
    full = B.Plan(cfg, 1 << 40, plan_tokens)
    fs = full.summary()
    attn_b = sum(s.bytes for s in full.shards() if s.kind in (B.PS_SHARD_QKV, B.PS_SHARD_O))
    tight = fs.workspace_bytes + 2 * B.Plan(cfg, fs.workspace_bytes + fs.weight_bytes - 4096, plan_tokens).summary().slot_bytes + 4096
    path = sorted({0} | set(rng.choice(n, size=min(n, 4), replace=False).tolist()))
    dpath = torch.tensor(path + [-1] * (n - len(path)), dtype=torch.int32, device="cuda:0")
    dcount = torch.tensor([len(path)], dtype=torch.int32, device="cuda:0")
    got = []
    for budget in (1 << 30, tight):
        st = _stack(cfg, W, plan_tokens, ctx, caches, budget)
        st.set_rotation(_inv_freq(st.device), norm=True)
        pinned = [s for s in st.plan.shards() if s.kind == B.PS_SHARD_KV and s.resident == 1]
        st.set_tree(parents)
        out = _forward(st, x)
        qkv = st.debug_buffer(0, np.float16, (n, rows, 128)).copy()
        attn = st.debug_buffer(5, np.float16, (n, n_q, 128)).copy()
        _check_rows(cfg, qkv, attn, caches[0][0], caches[0][1], ctx, parents)
        K, V = np.zeros((n_kv, cfg["kv_context"], 128), np.float16), np.zeros((n_kv, cfg["kv_context"], 128), np.float16)
        K[:, :ctx], V[:, :ctx] = caches[0]
        K[:, ctx:ctx + n], V[:, ctx:ctx + n] = qkv[:, n_q:n_q + n_kv].transpose(1, 0, 2), qkv[:, n_q + n_kv:].transpose(1, 0, 2)
        held = lambda s: st.arena[s.offset:s.offset + 2 * cfg["kv_context"] * 256].cpu().numpy().view(np.float16).reshape(2, -1, 128)  # noqa: E731
        for s in pinned:
            h = held(s)
            assert np.array_equal(h[0, :ctx + n].view(np.uint16), K[s.expert, :ctx + n].view(np.uint16))
            assert np.array_equal(h[1, :ctx + n].view(np.uint16), V[s.expert, :ctx + n].view(np.uint16))
        st.keep_path(dpath, dcount)
        with pytest.raises(B.PshardError):
            st.keep_path(dpath, dcount)                 # once
        for A in (K, V):
            A[:, ctx:ctx + len(path)] = A[:, [ctx + p for p in path]].copy()
        st.synchronize()
        for s in pinned:
            h = held(s)
            assert np.array_equal(h[0, :ctx + n].view(np.uint16), K[s.expert, :ctx + n].view(np.uint16))
            assert np.array_equal(h[1, :ctx + n].view(np.uint16), V[s.expert, :ctx + n].view(np.uint16))
        # the next step: the same tree behind the kept rows
        ctx2 = ctx + len(path)
        st.set_context(ctx2)
        out2 = _forward(st, x2)
        qkv2 = st.debug_buffer(0, np.float16, (n, rows, 128)).copy()
        attn2 = st.debug_buffer(5, np.float16, (n, n_q, 128)).copy()
        _check_rows(cfg, qkv2, attn2, K, V, ctx2, parents)
        got.append((out.cpu(), out2.cpu(), qkv, attn, attn2))
        if budget == tight and ctx >= 200 and n_kv > 1:
            assert len(pinned) < n_kv
        st.close()
    for a, b in zip(got[0], got[1]):
        a, b = np.asarray(a), np.asarray(b)
        assert np.array_equal(a.view(np.uint16), b.view(np.uint16))


@pytest.mark.parametrize("moe", [False, True])
def test_a_chain_as_a_tree_is_a_chunk(moe):
    """A chain gives what a chunk of the same tokens gives, within what fp16 weights differ by; rows that a tree leaves out of the plan are not touched."""
    import torch
    from paper_2604_26334_amd import binding as B
    cfg = _cfg(n_layers=2, cap=200, n_q=4, n_kv=1 if moe else 2, moe=moe)
    W, caches, n, M = Hn.WeightCache(cfg, 35), _caches(cfg, 35, 90), 11, 16
    x = S.activations(35, 0, n, cfg["hidden"])
    lg = S.router_logits(35, 0, 2, n, cfg["n_experts"]) if moe else None
    st = _stack(cfg, W, M, 90, caches)
    st.set_rotation(_inv_freq(st.device), norm=True)
    xin, xout = _tensors(st, x)
    B.chunked_forward(st, xin, xout, lg)
    st.synchronize()
    st.set_tree([i - 1 for i in range(n)])
    st.set_context(90)
    wide = torch.full((M, cfg["hidden"]), 7.0, dtype=torch.float16, device=st.device)
    torch.cuda.synchronize()
    st.forward(xin, wide[:n], lg)
    st.synchronize()
    assert bool((wide[n:] == 7).all())
    # both sides round weights and rows to fp16 (2^-11): two layers of about ten such steps each stay within 20 x 2^-11 of the largest value
    assert Hn.rel_err(wide[:n].cpu().numpy(), xout.cpu().numpy()) <= 20 * 2.0 ** -11
    st.close()


def test_a_tree_answers_as_decode_does_token_by_token():
    """Three layers with positions: every node's hidden state is that of decoding its ancestors one by one, and after keeping a path both caches go on alike."""
    cfg = _cfg(n_layers=3, cap=300)
    W, ctx, n = Hn.WeightCache(cfg, 37), 120, 9
    caches = _caches(cfg, 37, ctx)
    parents = [-1, 0, 0, 1, 1, 2, 3, 5, 6]
    x, nxt = S.activations(37, 0, n, cfg["hidden"]), S.activations(37, 1, 1, cfg["hidden"])
    tree = _stack(cfg, W, n, ctx, caches)
    one = _stack(cfg, W, 1, ctx, caches)
    for st in (tree, one):
        st.set_rotation(_inv_freq(st.device), norm=True)
    tree.set_tree(parents)
    got = _forward(tree, x).cpu().numpy()
    line = [0, 1, 3, 6, 8]
    for i, node in enumerate(line):
        one.set_context(ctx + i)
        want = _forward(one, x[node:node + 1]).cpu().numpy()
        # fp16 rows on both sides, scores of up to 11 whose rounded keys and queries move them by 2 x 11 x 2^-11: a weight by 1 %, a row by less than twice that
        assert Hn.rel_err(got[node:node + 1], want) <= 2e-2, node
    import torch
    tree.keep_path(torch.tensor(line + [-1] * 4, dtype=torch.int32, device="cuda:0"), torch.tensor([5], dtype=torch.int32, device="cuda:0"))
    tree.set_context(ctx + 5)
    one.set_context(ctx + 5)
    tree.set_tree([-1])
    assert Hn.rel_err(_forward(tree, nxt).cpu().numpy(), _forward(one, nxt).cpu().numpy()) <= 2e-2
    tree.close()
    one.close()


@pytest.mark.parametrize("drafts,temperature", [(True, 0.8), (False, 1.0), (True, 0.0), (False, None)])
def test_a_step_verifies_its_drafts_and_keeps_them(drafts, temperature):
    """Several steps of a loop as a user writes it, all of a step enqueued before one wait: what is accepted follows from the stack's own logits by the
    oracle's rule, and the cache's rows are the accepted tokens'."""
    import torch
    from paper_2604_26334_amd import binding as B
    V, n, ctx = 400, 8, 60
    cfg = _cfg(n_layers=2, cap=200, vocab=V)
    W, caches, head = Hn.WeightCache(cfg, 39), _caches(cfg, 39, ctx), S.head_matrix(39, cfg)
    st = _stack(cfg, W, n, ctx, caches, head=head)
    st.set_rotation(_inv_freq(st.device), norm=True)
    parents = [-1, 0, 0, 1, 1, 2, 3, 6]
    st.set_tree(parents)
    logits = torch.zeros(n, V, dtype=torch.float16, device=st.device)
    st.set_logits_out(logits, 0, n)
    rng = np.random.default_rng(3)
    embed = (rng.normal(size=(V, cfg["hidden"])) * 0.5).astype(np.float16)
    token0, sizes = 5, []
    for step in range(5):
        first = _forward(st, embed[[token0] + [0] * (n - 1)])         # (node 0's logits, to draw likely drafts from; its rows are overwritten below)
        near = logits.float().cpu().numpy()
        token = [token0] + [int(t) for t in np.argsort(-near[0], kind="stable")[:n - 1]]
        draft = (near * 0.9 + rng.normal(size=near.shape) * 0.3).astype(np.float16)
        dt = torch.tensor(token, dtype=torch.int32, device=st.device)
        u, us = (torch.tensor(rng.random(k) * (0.3 if k > 1 else 1.0), dtype=torch.float32, device=st.device) for k in (n, 1))
        dd = torch.from_numpy(draft).to(st.device) if drafts else None
        te = None if temperature is None else torch.tensor([temperature], dtype=torch.float32, device=st.device)
        xin, xout = _tensors(st, embed[token])
        torch.cuda.synchronize()
        st.forward(xin, xout)
        path, count, nxt = st.verify_tree(dt, u, us, draft_logits=dd, temperature=te, max_children=3)
        st.keep_path(path, count)
        st.synchronize()
        want, w_next = D.verify_tree(logits.double().cpu().numpy(), token, parents, u.tolist(), float(us[0]), draft.astype(np.float64) if drafts else None,
                                     1.0 if temperature is None else float(te[0]))
        k = int(count[0])
        assert path.tolist() == want + [-1] * (n - len(want)) and k == len(want) and int(nxt[0]) == w_next
        qkv = st.debug_buffer(0, np.float16, (n, 8, 128))         # the last layer's rows
        kv = [s for s in st.plan.shards() if s.kind == B.PS_SHARD_KV and s.layer == 1]
        for s in kv:
            h = st.arena[s.offset:s.offset + 2 * 200 * 256].cpu().numpy().view(np.float16).reshape(2, -1, 128)
            assert np.array_equal(h[0, ctx:ctx + k].view(np.uint16), qkv[want, 4 + s.expert].view(np.uint16))
            assert np.array_equal(h[1, ctx:ctx + k].view(np.uint16), qkv[want, 6 + s.expert].view(np.uint16))
        ctx, token0 = ctx + k, int(nxt[0])
        sizes.append(k)
        st.set_context(ctx)
        del first
    assert max(sizes) > 1
    # one token's logits: the draw of the next token alone
    st.set_logits_out(logits[:1].contiguous(), 3, 1)
    one = torch.zeros(V, dtype=torch.float16, device=st.device)
    st.set_logits_out(one, 3, 1)
    _forward(st, embed[token])
    path, count, nxt = st.verify_tree(dt[:1].contiguous(), u[:1].contiguous(), us, temperature=te)
    st.synchronize()
    want, w_next = D.verify_tree(one.double().cpu().numpy()[None], token[:1], [-1], [0.0], float(us[0]), None, 1.0 if temperature is None else float(te[0]))
    assert path.tolist() == [0] and int(count[0]) == 1 and int(nxt[0]) == w_next
    st.close()


def test_what_a_stack_refuses():
    import torch
    from paper_2604_26334_amd import binding as B
    L = B.lib()
    cfg = _cfg(cap=64, vocab=64)
    W, caches = Hn.WeightCache(cfg, 41), _caches(cfg, 41, 10)
    st = _stack(cfg, W, 8, 10, caches, head=S.head_matrix(41, cfg))

    def refused(code, call, *args):
        with pytest.raises(B.PshardError) as e:
            call(*args)
        assert e.value.code == code, e.value
    for bad in ([0], [-1, 1], [-1, 0, 5], [-2], [-1] * 9):
        refused(B.PS_E_ARG, st.set_tree, bad)
    path, count = torch.zeros(8, dtype=torch.int32, device=st.device), torch.ones(1, dtype=torch.int32, device=st.device)
    refused(B.PS_E_STATE, st.keep_path, path, count)                          # no forward yet
    dt, u = torch.zeros(8, dtype=torch.int32, device=st.device), torch.zeros(8, device=st.device)
    refused(B.PS_E_STATE, st.verify_tree, dt, u, u[:1])                       # no logits
    for kw in (dict(rot_dim=24), dict(rot_dim=256), dict(rot_dim=64, pairs=2), dict(rot_dim=64, norm=2), dict(rot_dim=64, inv_freq=None), dict(norm=1, q_gain=3)):
        a = dict(rot_dim=0, pairs=0, norm=0, reserved=0, inv_freq=1 << 30, q_gain=None, k_gain=None)
        a.update(kw)
        r = B.ps_rotation(**a)
        assert L.ps_stack_set_rotation(st.h, C.byref(r)) == B.PS_E_ARG
    assert L.ps_stack_set_tree(None, None, 0) == B.PS_E_ARG and L.ps_stack_set_tree(st.h, None, 3) == B.PS_E_ARG
    assert L.ps_stack_keep_path(st.h, None, None) == B.PS_E_ARG and L.ps_stack_set_rotation(None, None) == B.PS_E_ARG
    x = S.activations(41, 0, 5, cfg["hidden"])
    st.set_tree([-1, 0, 0, 1, 2])
    xin, xout = _tensors(st, x)
    refused(B.PS_E_STATE, B.chunked_forward, st, xin, xout)
    st.set_context(60)
    refused(B.PS_E_STATE, st.forward, xin, xout)                              # no room for the tree's rows
    st.set_context(59)
    _forward(st, x)
    st.keep_path(path[:5].contiguous(), count)
    st.close()
    plain = dict(Hn.small_dense_cfg(1))
    st = B.Stack(B.Plan(plain, 1 << 30, 8))
    refused(B.PS_E_STATE, st.set_tree, [-1, 0])
    refused(B.PS_E_STATE, st.set_rotation, torch.ones(64, device="cuda:0"))
    assert L.ps_stack_keep_path(st.h, 1 << 30, 1 << 30) == B.PS_E_STATE
    st.close()
    st = B.Stack(B.Plan(_cfg(cap=64), 1 << 30, 1))
    refused(B.PS_E_STATE, st.set_tree, [-1])
    st.close()
