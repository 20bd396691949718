"""Operators of a step that answers several drafted tokens, without a GPU: what the entry points refuse, and the oracle
against what the definitions fix."""
import ctypes as C

import numpy as np
import pytest

from oracle import drafts as D
from paper_2604_26334_amd import binding as B

PTR = 1 << 40          # an address that nobody reads: the calls below are refused before a launch


def _rope(**kw):
    a = dict(type=0, n_tokens=3, n_q_heads=4, n_k_heads=2, head_dim=128, rot_dim=128, pairs=0, norm=1, eps=1e-6, reserved=0,
             q=PTR, k=PTR + 65536, q_out=PTR, k_out=PTR + 65536, q_token=768, q_head=128, k_token=768, k_head=128,
             q_out_token=768, q_out_head=128, k_out_token=768, k_out_head=128, q_gain=None, k_gain=None, positions=PTR, inv_freq=PTR)
    a.update(kw)
    return B.ps_qk_norm_rope_args(**a)


def _tree(**kw):
    a = dict(type=0, n_seq=2, n_tokens=9, n_q_heads=4, n_kv_heads=2, head_dim=128, max_context=100, max_tree=8, capacity=128, append=0,
             scale=0.1, reserved=0, q=PTR, k_new=PTR, v_new=PTR, k_cache=PTR, v_cache=PTR, out=PTR + (1 << 20), q_token=1024, q_head=128,
             k_new_token=1024, k_new_head=128, v_new_token=1024, v_new_head=128, k_seq=65536, k_head=32768, k_row=128, v_seq=65536,
             v_head=32768, v_row=128, out_token=512, out_head=128, first=PTR, context=PTR, parent=PTR)
    a.update(kw)
    return B.ps_tree_attention_args(**a)


def _verify(**kw):
    a = dict(type=0, n_seq=2, n_tokens=9, vocab=1000, max_tree=8, max_children=3, target_logits=PTR, draft_logits=PTR, target_row=1000,
             draft_row=1000, path_seq=8, first=PTR, token=PTR, parent=PTR, u_accept=PTR, u_sample=PTR, temperature=None, path=PTR, count=PTR,
             next_token=PTR)
    a.update(kw)
    return B.ps_verify_tree_args(**a)


def _keep(**kw):
    a = dict(n_seq=2, n_planes=4, capacity=64, row_bytes=256, max_tree=8, reserved=0, cache=PTR, seq_stride=65536, plane_stride=16384,
             row_stride=256, path_seq=8, path=PTR, count=PTR, context=PTR)
    a.update(kw)
    return B.ps_cache_keep_args(**a)


def _refused(rc):
    assert rc == B.PS_E_ARG, rc
    assert B.lib().ps_last_error()


@pytest.mark.parametrize("kw", [
    dict(type=3), dict(head_dim=0), dict(head_dim=513), dict(rot_dim=3), dict(rot_dim=130), dict(pairs=2), dict(norm=2),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None),
    dict(q=PTR + 1), dict(q_out=PTR + 65536 * 2 + 1), dict(q_gain=PTR + 1), dict(k_gain=PTR + 1), dict(type=2, k=PTR + 2, k_out=PTR + 2),
    dict(q_out_token=1024), dict(k_out_head=256), dict(positions=None), dict(inv_freq=None), dict(positions=PTR + 2),
    dict(n_tokens=1 << 31), dict(n_tokens=1 << 30, n_q_heads=64), dict(n_q_heads=1 << 16)])
def test_rope_refuses(kw):
    _refused(B.lib().ps_qk_norm_rope(C.byref(_rope(**kw)), None))


@pytest.mark.parametrize("kw", [
    dict(type=2), dict(head_dim=96), dict(head_dim=0), dict(n_kv_heads=0), dict(n_q_heads=5), dict(n_q_heads=0), dict(n_q_heads=2048),
    dict(max_tree=257), dict(n_seq=1 << 16), dict(max_context=129), dict(append=1, max_context=121), dict(n_tokens=1 << 31),
    dict(q=None), dict(out=None), dict(k_cache=None), dict(first=None), dict(context=None), dict(parent=None), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(q=PTR + 8), dict(v_cache=PTR + 2), dict(q_token=1028), dict(k_row=129), dict(v_seq=4), dict(out_head=132),
    dict(k_row=1 << 25), dict(v_new_token=1 << 25), dict(first=PTR + 2)])
def test_tree_attention_refuses(kw):
    big = 1 << 40
    _refused(B.lib().ps_tree_attention(C.byref(_tree(**kw)), PTR, big, None))


@pytest.mark.parametrize("kw", [
    dict(type=3), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(max_tree=257), dict(max_children=0), dict(max_children=257), dict(n_seq=1 << 16),
    dict(n_tokens=1 << 31), dict(target_logits=None), dict(token=None), dict(parent=None), dict(u_accept=None), dict(u_sample=None), dict(first=None),
    dict(path=None), dict(count=None), dict(next_token=None), dict(path_seq=7), dict(target_logits=PTR + 1), dict(type=2, draft_logits=PTR + 2),
    dict(temperature=PTR + 1), dict(token=PTR + 2)])
def test_verify_refuses(kw):
    _refused(B.lib().ps_verify_tree(C.byref(_verify(**kw)), PTR, 1 << 40, None))


@pytest.mark.parametrize("kw", [
    dict(row_bytes=0), dict(row_bytes=24), dict(row_bytes=4112), dict(max_tree=257), dict(n_seq=1 << 16), dict(cache=None), dict(path=None),
    dict(count=None), dict(context=None), dict(cache=PTR + 8), dict(seq_stride=24), dict(plane_stride=8), dict(row_stride=264), dict(row_stride=240),
    dict(path=PTR + 1)])
def test_keep_refuses(kw):
    _refused(B.lib().ps_cache_keep(C.byref(_keep(**kw)), None))


def test_null_arguments_are_refused():
    L = B.lib()
    n = C.c_uint64()
    for rc in (L.ps_qk_norm_rope(None, None), L.ps_tree_attention(None, None, 0, None), L.ps_tree_attention_workspace(None, C.byref(n)),
               L.ps_tree_attention_workspace(C.byref(_tree()), None), L.ps_verify_tree(None, None, 0, None),
               L.ps_verify_tree_workspace(None, C.byref(n)), L.ps_verify_tree_workspace(C.byref(_verify()), None), L.ps_cache_keep(None, None)):
        _refused(rc)


def test_short_or_unaligned_workspaces_are_refused():
    L = B.lib()
    n = C.c_uint64()
    big = _tree(max_context=100000, capacity=100128)
    assert L.ps_tree_attention_workspace(C.byref(big), C.byref(n)) == 0
    if n.value:
        _refused(L.ps_tree_attention(C.byref(big), PTR, n.value - 1, None))
        _refused(L.ps_tree_attention(C.byref(big), None, n.value, None))
        _refused(L.ps_tree_attention(C.byref(big), PTR + 16, n.value, None))
    v = _verify(vocab=100000, target_row=100000, draft_row=100000)
    assert L.ps_verify_tree_workspace(C.byref(v), C.byref(n)) == 0
    if n.value:
        _refused(L.ps_verify_tree(C.byref(v), PTR, n.value - 1, None))
        _refused(L.ps_verify_tree(C.byref(v), None, n.value, None))
        _refused(L.ps_verify_tree(C.byref(v), PTR + 16, n.value, None))


def test_calls_with_nothing_to_do_return():
    L = B.lib()
    assert L.ps_qk_norm_rope(C.byref(_rope(n_tokens=0, q=None, k=None)), None) == 0
    assert L.ps_qk_norm_rope(C.byref(_rope(n_q_heads=0, n_k_heads=0)), None) == 0
    assert L.ps_tree_attention(C.byref(_tree(n_seq=0)), None, 0, None) == 0
    assert L.ps_tree_attention(C.byref(_tree(n_tokens=0)), None, 0, None) == 0
    assert L.ps_tree_attention(C.byref(_tree(max_tree=0)), None, 0, None) == 0
    assert L.ps_verify_tree(C.byref(_verify(n_seq=0)), None, 0, None) == 0
    for kw in (dict(n_seq=0), dict(n_planes=0), dict(max_tree=0), dict(capacity=0)):
        assert L.ps_cache_keep(C.byref(_keep(**kw)), None) == 0


def test_the_binding_refuses_what_it_can_see():
    import torch
    f16 = torch.float16
    q, k = torch.zeros(3, 4, 128, dtype=f16), torch.zeros(3, 2, 128, dtype=f16)
    pos, inv = torch.zeros(3, dtype=torch.int32), torch.zeros(64)
    for args, kw in [((q, k.float(), pos, inv), {}), ((q, k[:2], pos, inv), {}), ((q, k, pos.long(), inv), {}), ((q, k, pos[:2], inv), {}),
                     ((q, k, pos, None), {}), ((q, k, None, inv), {}), ((q.double(), k.double(), pos, inv), {}), ((q[0], k, pos, inv), {}),
                     ((q, k, pos, inv), dict(q_gain=torch.zeros(64, dtype=f16))), ((q.transpose(1, 2), k, pos, inv), {}),
                     ((q, k, pos, inv), dict(q_out=torch.zeros(3, 4, 64, dtype=f16))),
                     ((q, k, pos, inv), {})]:           # the last: tensors that are not on a GPU
        with pytest.raises(B.PshardError):
            B.qk_norm_rope(*args, **kw)
    lg = torch.zeros(3, 10)
    i3, first, u = torch.zeros(3, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32), torch.zeros(3)
    for args, kw in [((lg, i3, i3, first, u, u[:1]), {}), ((lg, i3.long(), i3, first, u, u[:1]), {}), ((lg, i3, i3, first[:1], u, u[:1]), {}),
                     ((lg, i3, i3, first, u.double(), u[:1]), {}), ((lg, i3, i3, first, u, u[:1]), dict(draft_logits=lg.half())),
                     ((lg, i3, i3, first, u, u[:1]), dict(temperature=u)), ((lg[0], i3, i3, first, u, u[:1]), {})]:
        with pytest.raises(B.PshardError):
            B.verify_tree(*args, **kw)
    cache = torch.zeros(1, 2, 8, 64, dtype=f16)
    p, one = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for args in [(cache, p, one, one), (cache[0], p, one, one), (cache, p.long(), one, one), (cache, p, p[0], one), (cache.transpose(2, 3), p, one, one)]:
        with pytest.raises(B.PshardError):
            B.cache_keep(*args)
    kc = torch.zeros(1, 2, 16, 128, dtype=f16)
    par = torch.zeros(3, dtype=torch.int32)
    for bad in (dict(q=q.float()), dict(k_new=k[:, :1]), dict(v_cache=kc[:, :, :8]), dict(first=first.long()), dict(parent=par[:2]), dict()):
        a = dict(q=q, k_new=k, v_new=k, k_cache=kc, v_cache=kc, first=first, context=one, parent=par)
        a.update(bad)
        with pytest.raises(B.PshardError):
            B.tree_attention(**a, max_context=8, max_tree=3)


# ------------------------------------------------------------------ the oracle

def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(0)
    t, hq, hk, d, ctx = 6, 4, 2, 64, 11
    q, kn, vn = rng.normal(size=(t, hq, d)), rng.normal(size=(t, hk, d)), rng.normal(size=(t, hk, d))
    kc, vc = rng.normal(size=(hk, 20, d)), rng.normal(size=(hk, 20, d))
    got = D.tree_attention(q, kn, vn, kc, vc, ctx, [i - 1 for i in range(t)], d ** -0.5)
    for h in range(hq):
        k = np.concatenate([kc[h // 2, :ctx], kn[:, h // 2]])
        v = np.concatenate([vc[h // 2, :ctx], vn[:, h // 2]])
        for i in range(t):
            z = (k[:ctx + i + 1] @ q[i, h]) * d ** -0.5
            w = np.exp(z - z.max())
            assert np.allclose(got[i, h], (w / w.sum()) @ v[:ctx + i + 1], atol=1e-12)


def test_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(1)
    inv = np.exp(-np.arange(32) / 32 * np.log(10000.0)).astype(np.float32)
    x = rng.normal(size=(2, 1, 64))
    for pairs in (False, True):
        a = D.qk_norm_rope(np.repeat(x[:1], 4, 0), None, [3, 10, 1003, 1010], inv, 0, False, pairs)
        b = D.qk_norm_rope(np.repeat(x[1:], 4, 0), None, [5, 12, 1005, 1012], inv, 0, False, pairs)
        dots = (a * b).sum((1, 2))
        assert np.allclose(dots, dots[0], atol=1e-9)             # a product depends on the difference of the positions alone
        assert np.allclose((a * a).sum((1, 2)), (x[:1] ** 2).sum(), atol=1e-9)


@pytest.mark.parametrize("drafts,shape", [(True, "chain"), (True, "two"), (True, "three"), (False, "two")])
def test_verified_tokens_are_distributed_as_the_targets(drafts, shape):
    """The first token behind node 0, accepted draft or drawn in its place, has the target's distribution."""
    rng = np.random.default_rng(2)
    V, T, N = 5, 0.7, 20000
    target = rng.normal(size=(4, V)) * 1.5
    draft = rng.normal(size=(4, V)) * 1.5
    m = {"chain": 1, "two": 2, "three": 3}[shape]
    parent = [-1] + [0] * m
    p, q = D._row(target[0], T), D._row(draft[0], T)
    seen = np.zeros(V)
    for _ in range(N):
        token = [0] + list(rng.choice(V, size=m, p=q) if drafts else np.argsort(-draft[0])[:m])
        path, nxt = D.verify_tree(target[:m + 1], token, parent, rng.random(m + 1), rng.random(), draft[:m + 1] if drafts else None, T)
        seen[token[path[1]] if len(path) > 1 else nxt] += 1
    # a frequency of N draws is off by 5 standard deviations once in 1.7 million times
    assert np.all(np.abs(seen / N - p) < 5 * np.sqrt(p * (1 - p) / N)), (seen / N, p)
