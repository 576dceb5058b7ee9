"""Calls of the paged 4-bit cache at the edges of what its header allows:
arguments that are the cache's own buffers.  Against the plain model of
tests/pagedref.py."""
import numpy as np
import pytest

from tests import pagedref as R
from tests.test_gpu_paged import assert_tables, fill, ints, make, starts_of

pytestmark = pytest.mark.gpu


def model_of(c):
    """The plain model of the cache's present tables."""
    m = R.Pages(c.cfg.n_pages, c.cfg.max_seqs, c.cfg.seq_pages)
    m.lens = c.lens.cpu().tolist()
    m.rows = [row[:-(-n // 64)] for row, n in zip(c.table.cpu().tolist(), m.lens)]
    return m


# ------------------------------------------------- the cache's own buffers --

def test_assign_takes_the_caches_own_tables():
    """Its own lengths and tables change nothing; shorter lengths over its own
    tables drop tokens, its own lengths with another table replace pages."""
    import torch
    rng = np.random.default_rng(50)
    c = make(n_pages=20, seqs=4, seq_pages=6)
    fill(c, [200, 90, 0, 64], rng)
    c.fork(ints([0, 1, 1, 3]))                           # a page that two slots hold
    lens, m = [200, 90, 90, 64], model_of(c)
    before = c.read(0, starts_of(lens), sum(lens))
    c.assign(c.lens, c.table)
    assert_tables(c, m)
    assert all(torch.equal(a, b) for a, b in zip(before, c.read(0, starts_of(lens), sum(lens))))
    short = [130, 64, 90, 0]
    c.assign(ints(short), c.table)
    m.lens, m.rows = short, [r[:-(-n // 64)] for r, n in zip(m.rows, short)]
    assert_tables(c, m)
    other = c.table.clone()
    other[0, 1], other[3, 2] = 19, 7                     # the second is beyond its sequence's length
    c.assign(c.lens, other)
    m.rows[0][1] = 19
    assert_tables(c, m)
    assert c.status() == 0
    other[0, 0] = 20                                     # no such page
    c.assign(c.lens, other)
    m.rows[0][0] = -1
    assert_tables(c, m)
    assert c.status() == R.BAD_INDEX


def test_own_lengths_as_counts():
    """Lengths as what a call adds, keeps or takes as parents."""
    import torch
    c = make(n_pages=20, seqs=4, seq_pages=6)
    fill(c, [100, 2, 0, 3], np.random.default_rng(51))
    m = model_of(c)
    c.reserve(c.lens)
    m.reserve(list(m.lens))
    assert_tables(c, m)
    keep = torch.arange(200, dtype=torch.int32, device="cuda").repeat(4, 1)
    lens = list(m.lens)
    c.compact(keep, c.lens)
    m.compact(lens, 200)
    assert_tables(c, m)
    c.assign(ints([3, 1, 0, 2]), c.table)
    m.lens, m.rows = [3, 1, 0, 2], [r[:-(-n // 64)] for r, n in zip(m.rows, [3, 1, 0, 2])]
    c.fork(c.lens)
    m.fork([3, 1, 0, 2])
    assert_tables(c, m)
    assert c.status() == 0
