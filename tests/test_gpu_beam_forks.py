"""Reordering of rows of different lengths on the GPU: no row's next position lies in a page that another row still reads."""
import numpy as np
import pytest
import torch

from paper_2303_06865_amd import binding as B
from tests import plain_forks as F
from tests.util import dev, host

pytestmark = pytest.mark.gpu


def _pool(cfg, n_pages, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = B.KVPages(cfg, n_pages, int8=True)
    for t in (pages.k_codes, pages.v_codes):
        t.random_(-127, 128, generator=g)
    for t in (pages.k_meta, pages.v_meta):
        t.uniform_(0.01, 0.02, generator=g)
    return pages


def _rows(cfg, pages, table, pos):
    """What every row's sequence holds."""
    n = max(1, int(pos.max()))
    k, v = (host(t) for t in B.fg_kv_gather_paged(cfg, pages, B.Ragged(dev(table)), len(pos), n))
    return [(k[i, :pos[i]].copy(), v[i, :pos[i]].copy()) for i in range(len(pos))]


def _check(nh, dh, table, pos, parents, beams, per, inplace, seed):
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 4096)
    table, pos, parents = (np.array(a, np.int32) for a in (table, pos, parents))
    rows = len(pos)
    pages = _pool(cfg, rows // beams * per, seed)
    before = _rows(cfg, pages, table, pos)
    dt, dp = dev(table), dev(pos)
    kw = dict(table_out=dt, pos_out=dp) if inplace else {}
    got_t, got_p, miss = B.fg_beam_reorder_paged(cfg, [pages], dt, dp, dev(parents), beams, per, **kw)
    wt, wp, wm, _ = F.reorder(table, pos, parents, beams, per)
    assert np.array_equal(host(got_t), wt) and np.array_equal(host(got_p), wp) and np.array_equal(host(miss), wm)
    after = _rows(cfg, pages, wt, wp)
    held = [i for i in range(rows) if wp[i] % 64 == 0 or wt[i, wp[i] // 64] >= 0]     # a begun page without a place is lost
    for i in held:
        p = parents[i] if 0 <= parents[i] < beams else i % beams
        for a, b in zip(after[i], before[i // beams * beams + p]):
            assert np.array_equal(a, b), i
    # a row stored behind row i, large enough to be seen anywhere in its page, is seen by row i alone
    for i in range(rows):
        big = dev(np.full((1, 2 * nh * dh), 9.0, np.float16))
        B.fg_kv_append_paged(cfg, big, big[:, nh * dh:], 2 * nh * dh, 1, 1, pages,
                             B.Ragged(dev(wt), dev(np.array([i], np.int32)), dev(wp[i:i + 1])))
        now = _rows(cfg, pages, wt, wp)
        for j in held:
            if j > i:
                for a, b in zip(now[j], after[j]):
                    assert np.array_equal(a, b), (i, j)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("pos,parents", [([128, 70], [0, 1]), ([70, 128], [0, 1]), ([128, 70], [1, 0]), ([127, 192], [0, 1]),
                                         ([65, 192], [0, 1]), ([70, 192], [1, 1]), ([64, 192], [0, 1])])
def test_a_fork_from_an_earlier_position(pos, parents, inplace):
    """Both rows name pages 0, 1 (and 2): one of them still needs what the other would write to."""
    _check(2, 64, [[0, 1, 2, -1]] * 2, pos, parents, 2, 8, inplace, 1)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_random_forks(seed, inplace):
    r = np.random.default_rng(seed)
    beams, groups, stride = [(2, 3, 4), (16, 1, 6), (4, 2, 3), (5, 2, 8), (8, 2, 5), (3, 1, 300)][seed]
    per = beams * stride + beams
    table, pos = F.tree(r, groups, beams, stride, per)
    _check(1 + seed % 2, 64 if seed % 3 else 128, table, pos, r.integers(0, beams, groups * beams), beams, per, inplace, seed)


def test_without_a_free_page():
    """A row that may not keep its begun page and finds no other has none (-1), and is counted."""
    _check(2, 64, [[0, 1, -1], [0, 1, 2]], [70, 130], [0, 1], 2, 3, False, 3)
