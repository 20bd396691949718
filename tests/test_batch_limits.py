"""Operators of a batch of requests without a GPU: what they ask for, at the ends of their ranges."""
import ctypes as C

import pytest

from paper_2604_26334_amd import binding as B


def _workspace(**kw):
    n = C.c_uint64()
    a = B.ps_page_attention_args(page=16, n_pages=100000, scale=0.1, **kw)
    assert B.lib().ps_page_attention_workspace(C.byref(a), C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("seqs,most", [(1, 1), (3, 2), (64, 1), (64, 8), (48, 9), (8, 40)])
@pytest.mark.parametrize("length,prefix", [(32768, 0), (1000, 0), (1000, 200), (1000, 32761), (40, 32761)])
def test_room_for_more_tokens_than_may_be_answered_costs_nothing(seqs, most, length, prefix):
    """A captured step keeps rows for its largest batch: what a call needs, and into how many runs it cuts positions (a place holds one record of each), goes by
    the tokens that its sequences may have."""
    a = dict(type=0, head_dim=128, n_q_heads=32, n_kv_heads=8, n_seq=seqs, max_tokens=most, max_length=length, width=2048, n_prefix=1 if prefix else 0, max_prefix=prefix, prefix_width=2048)
    need = _workspace(n_tokens=seqs * most, **a)
    for n in (seqs * most + 1, 1024, 16384, 1 << 20):
        assert _workspace(n_tokens=n, **a) == need, n


def test_prefixes_without_a_bound_are_seen_whole(monkeypatch):
    """A prefix's length is bounded by its table's room where the caller names no bound, and by the caller's where there is one."""
    import torch
    seen = []
    monkeypatch.setattr(B, "_launch", lambda dev, call, args, *rest: seen.append(args._obj))
    i32, pages, q = torch.int32, torch.zeros(4, 2, 16, 64, dtype=torch.float16), torch.zeros(3, 4, 64, dtype=torch.float16)
    a = dict(q=q, k_pages=pages, v_pages=pages, first=torch.tensor([0, 3], dtype=i32), length=torch.zeros(1, dtype=i32), table=torch.zeros(1, 2, dtype=i32), max_length=16, max_tokens=3)
    behind = dict(group_first=torch.tensor([0, 1], dtype=i32), prefix_length=torch.zeros(1, dtype=i32), prefix_table=torch.zeros(1, 7, dtype=i32))
    for kw, want in ((behind, 7 * 16), (dict(behind, max_prefix=None), 7 * 16), (dict(behind, max_prefix=33), 33), (dict(behind, max_prefix=0), 0), ({}, 0)):
        B.page_attention(**a, **kw)
        assert seen[-1].max_prefix == want and seen[-1].n_prefix == (1 if kw else 0)
    with pytest.raises(B.PshardError):
        B.page_attention(**a, **behind, max_prefix=113)
