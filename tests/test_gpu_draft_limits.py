"""Operators of drafted tokens at sizes that one launch's threads do not cover."""
import numpy as np
import pytest

from oracle import drafts as D
from tests import test_gpu_drafts as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [16, 2])
def test_rope_of_more_heads_than_a_launch_holds(d):
    """2^26 + 1003 tokens of one head: rows at both ends and around 2^26 against the oracle, and the others' lengths (a row's norm is 1)."""
    import torch
    from paper_2604_26334_amd import binding as B
    n = (1 << 26) + 1003
    x = torch.empty(n, 1, d, dtype=torch.float16, device=T.DEV)
    for lo in range(0, n, 1 << 23):
        x[lo:lo + (1 << 23)].normal_(generator=T._gen(lo + 1))
    pos = torch.arange(n, dtype=torch.int32, device=T.DEV)
    inv = torch.tensor(np.exp(-np.arange(d // 2) / (d // 2) * np.log(10000.0)), dtype=torch.float32, device=T.DEV)
    spots = list(range(40)) + [(1 << 26) + i for i in range(-40, 40)] + list(range(n - 40, n)) + np.random.default_rng(1).integers(0, n, 200).tolist()
    at = torch.tensor(spots, device=T.DEV)
    before = T._np(x[at])
    got, _ = B.qk_norm_rope(x, x[:, :0], pos, inv, q_out=x, k_out=x[:, :0])
    ref = D.qk_norm_rope(before, None, spots, inv.cpu().numpy(), 1e-6, True, False)
    off = np.abs(T._np(got[at]) - ref) / T._rope_tolerance(before, inv.cpu().numpy(), spots, ref, True, "f16")
    assert off.max() <= 1, off.max()
    for lo in range(0, n, 1 << 23):
        sizes = got[lo:lo + (1 << 23)].float().square().mean(-1)
        # (each value rounded to fp16: 2^-11 of it, twice that of its square; rows of small numbers fall behind by eps)
        assert bool((sizes <= 1 + 2.0 ** -9).all()) and float((sizes >= 1 - 2.0 ** -9).float().mean()) > 0.9
