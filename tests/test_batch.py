"""Operators of a step that answers a batch of requests over one paged cache, without a GPU: what the entry points refuse, and the
oracle against what the definitions fix."""
import ctypes as C

import numpy as np
import pytest

from oracle import batch as O
from paper_2604_26334_amd import binding as B

PTR = 1 << 40          # an address that nobody reads: the calls below are refused before a launch


def _tables(**kw):
    a = dict(n_seq=3, n_tokens=9, page=16, width=8, n_pages=100, n_free=50, cached=PTR, new_tokens=PTR, offset=None, free_pages=PTR, free_at=PTR,
             table=PTR, table_seq=8, first=PTR, length=PTR, position=PTR, slot=PTR, taken=PTR)
    a.update(kw)
    return B.ps_page_tables_args(**a)


def _append(**kw):
    a = dict(n_tokens=5, n_heads=2, row_bytes=256, page=16, n_pages=10, reserved=0, k=PTR, v=PTR, k_pages=PTR, v_pages=PTR, k_token=512, k_head=256,
             v_token=512, v_head=256, k_page=8192, k_page_head=4096, k_page_row=256, v_page=8192, v_page_head=4096, v_page_row=256, slot=PTR)
    a.update(kw)
    return B.ps_page_append_args(**a)


def _attend(**kw):
    a = dict(type=0, n_seq=2, n_tokens=9, n_q_heads=4, n_kv_heads=2, head_dim=128, page=16, n_pages=100, width=8, n_prefix=1, prefix_width=20,
             max_length=128, max_prefix=320, max_tokens=8, scale=0.1, reserved=0, q=PTR, k_pages=PTR, v_pages=PTR, out=PTR + (1 << 20), q_token=512,
             q_head=128, k_page=8192, k_head=2048, k_row=128, v_page=8192, v_head=2048, v_row=128, out_token=512, out_head=128, table_seq=8,
             prefix_seq=20, first=PTR, length=PTR, table=PTR, group_first=PTR, prefix_length=PTR, prefix_table=PTR)
    a.update(kw)
    return B.ps_page_attention_args(**a)


def _sample(**kw):
    a = dict(type=0, n_rows=3, vocab=1000, reserved=0, logits=PTR, logits_row=1000, u=PTR, temperature=None, top_k=None, top_p=None, min_p=None,
             token=PTR, kept=None)
    a.update(kw)
    return B.ps_sample_args(**a)


def _refused(rc):
    assert rc == B.PS_E_ARG, rc
    assert B.lib().ps_last_error()


@pytest.mark.parametrize("kw", [
    dict(page=0), dict(page=8), dict(page=24), dict(page=2048), dict(n_seq=8193), dict(n_tokens=(1 << 30) + 1), dict(n_pages=1 << 28), dict(cached=None),
    dict(new_tokens=None), dict(free_pages=None), dict(table=None), dict(table_seq=7), dict(first=None), dict(length=None), dict(slot=None),
    dict(taken=None), dict(cached=PTR + 2), dict(offset=PTR + 1), dict(free_at=PTR + 2), dict(position=PTR + 1), dict(slot=PTR + 3)])
def test_tables_refuse(kw):
    _refused(B.lib().ps_page_tables(C.byref(_tables(**kw)), None))


@pytest.mark.parametrize("kw", [
    dict(page=0), dict(page=17), dict(page=2048), dict(row_bytes=0), dict(row_bytes=24), dict(row_bytes=4112), dict(n_tokens=(1 << 30) + 1),
    dict(n_heads=65536), dict(n_pages=1 << 28), dict(k=None), dict(v=None), dict(k_pages=None), dict(v_pages=None), dict(slot=None), dict(k=PTR + 8),
    dict(v_pages=PTR + 4), dict(k_token=520), dict(v_head=8), dict(k_page=24), dict(v_page_row=264), dict(slot=PTR + 2)])
def test_append_refuses(kw):
    _refused(B.lib().ps_page_append(C.byref(_append(**kw)), None))


@pytest.mark.parametrize("kw", [
    dict(type=2), dict(head_dim=96), dict(head_dim=0), dict(n_kv_heads=0), dict(n_q_heads=5), dict(n_q_heads=0), dict(n_q_heads=2048), dict(page=8),
    dict(page=48), dict(page=2048), dict(n_seq=1 << 16), dict(n_tokens=1 << 31), dict(n_pages=1 << 31), dict(n_prefix=4097), dict(max_length=129),
    dict(max_prefix=321), dict(q=None), dict(out=None), dict(k_pages=None), dict(v_pages=None), dict(first=None), dict(length=None), dict(table=None),
    dict(group_first=None), dict(prefix_length=None), dict(prefix_table=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=PTR + 8),
    dict(v_pages=PTR + 2), dict(q_token=516), dict(k_row=129), dict(v_page=4), dict(out_head=132), dict(k_row=1 << 26), dict(v_row=1 << 27), dict(page=1024, width=2, v_row=1 << 21), dict(k_page=1 << 35), dict(v_page=1 << 36),
    dict(first=PTR + 2), dict(prefix_table=PTR + 1)])
def test_attention_refuses(kw):
    _refused(B.lib().ps_page_attention(C.byref(_attend(**kw)), PTR, 1 << 60, None))


@pytest.mark.parametrize("kw", [
    dict(type=3), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(n_rows=1 << 16), dict(logits=None), dict(u=None), dict(token=None), dict(logits=PTR + 1),
    dict(type=2, logits=PTR + 2), dict(u=PTR + 2), dict(temperature=PTR + 1), dict(top_k=PTR + 1), dict(top_p=PTR + 2), dict(min_p=PTR + 2),
    dict(token=PTR + 2), dict(kept=PTR + 2)])
def test_sample_refuses(kw):
    _refused(B.lib().ps_sample(C.byref(_sample(**kw)), PTR, 1 << 60, None))


def test_null_arguments_are_refused():
    L, n = B.lib(), C.c_uint64()
    for rc in (L.ps_page_tables(None, None), L.ps_page_append(None, None), L.ps_page_attention(None, None, 0, None),
               L.ps_page_attention_workspace(None, C.byref(n)), L.ps_page_attention_workspace(C.byref(_attend()), None), L.ps_sample(None, None, 0, None),
               L.ps_sample_workspace(None, C.byref(n)), L.ps_sample_workspace(C.byref(_sample()), None)):
        _refused(rc)


def test_short_or_unaligned_workspaces_are_refused():
    L, n = B.lib(), C.c_uint64()
    for need, call, a in ((L.ps_page_attention_workspace, L.ps_page_attention, _attend(max_prefix=100000, prefix_width=10000)),
                          (L.ps_sample_workspace, L.ps_sample, _sample(n_rows=9, vocab=100000, logits_row=100000))):
        assert need(C.byref(a), C.byref(n)) == 0
        if n.value:
            _refused(call(C.byref(a), PTR, n.value - 1, None))
            _refused(call(C.byref(a), None, n.value, None))
            _refused(call(C.byref(a), PTR + 16, n.value, None))


def test_empty_calls_need_nothing():
    """No tokens, sequences, heads, pages or rows: nothing to launch, nothing to point at."""
    L = B.lib()
    assert L.ps_page_append(C.byref(B.ps_page_append_args(page=16, row_bytes=16)), None) == 0
    assert L.ps_page_attention(C.byref(B.ps_page_attention_args(head_dim=64, page=16, n_kv_heads=1, n_q_heads=1)), None, 0, None) == 0
    assert L.ps_sample(C.byref(B.ps_sample_args(vocab=5)), None, 0, None) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    f16, i32 = torch.float16, torch.int32
    one, pages = torch.zeros(1, dtype=i32), torch.zeros(4, 2, 16, 64, dtype=f16)
    q, first = torch.zeros(3, 4, 64, dtype=f16), torch.tensor([0, 3], dtype=i32)
    for bad in (dict(q=q.float()), dict(v_pages=pages[:, :1]), dict(first=first.long()), dict(length=first), dict(table=one), dict(group_first=first),
                dict(out=q[:2]), dict()):
        a = dict(q=q, k_pages=pages, v_pages=pages, first=first, length=one, table=one[None])
        a.update(bad)
        with pytest.raises(B.PshardError):
            B.page_attention(**a, max_length=16, max_tokens=3)
    k = torch.zeros(3, 2, 64, dtype=f16)
    for bad in (dict(v=k[:2]), dict(k_pages=pages.float()), dict(slot=one), dict(v_pages=pages[:, :, :, :32]), dict()):
        a = dict(k=k, v=k, k_pages=pages, v_pages=pages, slot=torch.zeros(3, dtype=i32))
        a.update(bad)
        with pytest.raises(B.PshardError):
            B.page_append(**a)
    lg, u = torch.zeros(3, 50), torch.zeros(3)
    for bad in (dict(logits=lg[0]), dict(logits=lg.double()), dict(u=u[:2]), dict(temperature=u.half()), dict(top_k=u), dict(top_p=u[:1]), dict(token=one), dict()):
        with pytest.raises(B.PshardError):
            B.sample(**dict(dict(logits=lg, u=u), **bad))
    t = dict(cached=one, new_tokens=one, table=one[None], free_pages=first, free_at=one, page=16, n_pages=4, n_tokens=3)
    for bad in (dict(cached=one[None]), dict(new_tokens=first), dict(table=one), dict(free_at=first), dict(offset=first), dict(slot=one), dict(n_tokens=-1), dict()):
        with pytest.raises(B.PshardError):
            B.page_tables(**dict(t, **bad))


# ------------------------------------------------------------------ the oracle

def test_tables_by_hand():
    """Three sequences in pages of 16: one begins, one stays in its page, one needs two more."""
    table = [[-1, -1, -1], [7, -1, -1], [5, 6, -1]]
    got = O.page_tables([0, 3, 31], [2, 4, 20], table, [9, 8, 4, 3], 1, 16, 10, 40, offset=[100, 0, 5])
    assert got[0] == [[8, -1, -1], [7, -1, -1], [5, 6, 4]]        # the third page of 51 positions is there; a fourth would be behind the table
    assert got[1] == [0, 2, 6, 26] and got[2] == [2, 7, 51] and got[5] == 2
    assert got[3] == [100, 101, 3, 4, 5, 6] + list(range(36, 56))
    assert got[4] == [128, 129] + [7 * 16 + i for i in (3, 4, 5, 6)] + [6 * 16 + 15] + [4 * 16 + i for i in range(16)] + [-1] * 3


def test_attention_does_not_depend_on_how_positions_are_told_apart():
    """A prefix and own positions are one run of positions; pages in any order hold the same rows."""
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(2, 20, 8)), rng.normal(size=(2, 20, 8))
    got = O.attention(q, k, v, np.ones(20, bool), 17, 0.3)
    for i in range(3):
        for h in range(4):
            z = k[h // 2, :18 + i] @ q[i, h] * 0.3
            w = np.exp(z) / np.exp(z).sum()
            assert np.allclose(got[i, h], w @ v[h // 2, :18 + i], atol=1e-12)
    pages = rng.normal(size=(5, 2, 4, 8))
    rows, there = O.rows_of(pages, [3, 0, 9, -1], 14)
    assert there.tolist() == [True] * 8 + [False] * 6
    assert np.array_equal(rows[:, 0], pages[3, :, 0]) and np.array_equal(rows[:, 6], pages[0, :, 2])


def test_sampled_tokens_have_the_kept_distribution():
    rng = np.random.default_rng(1)
    x, T, N = rng.normal(size=12) * 2, 0.8, 40000
    for settings in (dict(), dict(top_k=5), dict(top_p=0.8), dict(min_p=0.1), dict(top_k=9, top_p=0.9, min_p=0.02)):
        at, total, n = O.kept(x, temperature=T, **settings)
        p = np.zeros(12)
        p[at[:n]] = np.exp(x[at[:n]] / T)
        p /= p.sum()
        seen = np.bincount([O.sample(x, u, temperature=T, **settings)[0] for u in rng.random(N)], minlength=12) / N
        # a frequency of N draws is off by 5 standard deviations once in 1.7 million times
        assert np.all(np.abs(seen - p) <= 5 * np.sqrt(p * (1 - p) / N)), settings


def test_what_is_kept():
    x = np.log([0.4, 0.1, 0.3, 0.1, 0.05, 0.05])
    for settings, want in ((dict(), 6), (dict(top_k=2), 2), (dict(top_k=9), 6), (dict(top_k=-1), 6), (dict(top_p=0.35), 1), (dict(top_p=0.65), 2), (dict(top_p=0.0), 1),
                           (dict(top_k=3, top_p=0.6), 2), (dict(min_p=0.24), 4), (dict(min_p=2.0), 1), (dict(temperature=0.0), 1),
                           (dict(top_p=float("nan")), 6), (dict(min_p=float("nan")), 6)):
        assert O.kept(x, **settings)[2] == want, settings
    assert O.sample([1.0, 3.0, 3.0, 2.0], 0.0, top_k=1) == (1, 1)            # the lower index first among equals
    assert O.sample([float("-inf")] * 3, 0.5) == (-1, 0) and O.sample([float("nan"), 0.0], 0.9) == (1, 1)
