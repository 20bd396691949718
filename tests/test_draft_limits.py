"""Calls of the operators of drafted tokens that one launch cannot hold are refused before it."""
import ctypes as C

import pytest

from paper_2604_26334_amd import binding as B
from tests import test_drafts as T


@pytest.mark.parametrize("kw", [
    dict(n_seq=65535, n_kv_heads=512, n_q_heads=512), dict(n_seq=65535, n_kv_heads=257, n_q_heads=257), dict(n_seq=65535, n_kv_heads=128, n_q_heads=1024, max_tree=48)])
def test_tree_attention_beyond_a_launch(kw):
    """A launch of 2^24 workgroups of 256 threads is one too many."""
    a = T._tree(**kw)
    n = C.c_uint64()
    assert B.lib().ps_tree_attention_workspace(C.byref(a), C.byref(n)) == 0
    T._refused(B.lib().ps_tree_attention(C.byref(a), T.PTR, 1 << 60, None))


@pytest.mark.parametrize("planes", [(1 << 26) - 3, 1 << 26, (1 << 31) - 1, (1 << 32) - 1])
def test_kept_rows_of_more_planes_than_a_launch_holds(planes):
    """Four planes to a workgroup of 256 threads."""
    T._refused(B.lib().ps_cache_keep(C.byref(T._keep(n_planes=planes)), None))
