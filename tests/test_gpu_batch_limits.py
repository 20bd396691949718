"""Operators of a batch of requests at the ends of their ranges."""
import numpy as np
import pytest

from tests.test_gpu_drafts import DEV, _ints, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cached,new", [
    ([0, 5], [2 ** 30, 2 ** 30]), ([2 ** 30, 2 ** 30, 7, 2 ** 30], [2 ** 29] * 4), ([3] * 70, [2 ** 31 - 1] * 70), ([2 ** 31 - 1, 2 ** 30 - 1], [1, 2 ** 30]),
    ([0] * 600, [2 ** 21 + 1] * 600), ([1, 2, 3], [2 ** 30 - 2, 1, 5])])
def test_tables_of_as_many_tokens_as_there_may_be(cached, new):
    """n_tokens of 2^30, and new tokens that come to it or to more: their sums end there, and nothing behind the arrays is written."""
    from paper_2604_26334_amd import binding as B
    torch, n, guard, page, width = _t(), 1 << 30, 1 << 20, 1024, 2
    seqs = len(cached)
    buf = torch.full((2, n + guard), -9, dtype=torch.int32, device=DEV)
    table, free = torch.full((seqs, width), 3, dtype=torch.int32, device=DEV), torch.arange(100, 100 + 2 * seqs, dtype=torch.int32, device=DEV)
    first, length, position, slot, taken = B.page_tables(_ints(cached), _ints(new), table, free, None, page=page, n_pages=5000, n_tokens=n, position=buf[0, :n],
                                                         slot=buf[1, :n])
    want_first, want_length, pages, rows = [0], [], 0, [[3] * width for _ in range(seqs)]
    for s in range(seqs):
        c = min(cached[s], 2 ** 30)
        t = min(new[s], n - want_first[-1])
        want_first.append(want_first[-1] + t)
        want_length.append(min(c + t, 2 ** 30))
        for entry in range(min(width, -(-c // page)), min(width, -(-want_length[-1] // page))):
            rows[s][entry] = 100 + pages
            pages += 1
    assert first.tolist() == want_first and length.tolist() == want_length and int(taken) == pages and table.tolist() == rows
    total = want_first[-1]
    assert bool((buf[:, total:] == -9).all())
    at = np.unique(np.concatenate([np.clip(np.array(want_first)[:, None] + np.arange(-3, 2051), 0, total - 1).ravel(), np.linspace(0, total - 1, 1001).astype(np.int64)]))
    s = np.searchsorted(np.array(want_first[1:]), at, side="right")
    j = np.minimum(np.array(cached), 2 ** 30)[s] + at - np.array(want_first)[s]
    there = torch.from_numpy(at).to(DEV)
    assert np.array_equal(position[there].cpu().numpy(), j.astype(np.int32))
    entry = np.minimum(j // page, width - 1)
    assert np.array_equal(slot[there].cpu().numpy(), np.where(j // page < width, np.array(rows)[s, entry] * page + j % page, -1))
