"""Selections in which many continuations reach the bound of the best, and the largest calls that selection and reordering take."""
import numpy as np
import pytest
import torch

from paper_2303_06865_amd import binding as B
from tests import plain_forks as F
from tests.test_gpu_beam import _check_select
from tests.util import dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [50272, 50271, 20000])
@pytest.mark.parametrize("n,beams,n_best", [(1, 4, 32), (2, 16, 32), (1, 1, 32), (3, 8, 16), (1, 16, 8), (128, 4, 32)])
def test_select_of_many_near_the_best(vocab, n, beams, n_best):
    """Beams of equal scores over rows of one kind: the second pass has some hundred pieces with a good word each, of which more
    reach its bound than it lists."""
    if n > 100 and vocab != 50272:
        vocab = 5000
    r = np.random.default_rng(vocab)
    x = (r.standard_normal((n * beams, vocab)) * 2).astype(np.float32)
    _check_select(x, np.zeros(n * beams, np.float32), beams, n_best)
    _check_select(x, np.zeros(n * beams, np.float32), beams, n_best, (r.random(n * beams) < 0.3).astype(np.int32), eos=1)


@pytest.mark.parametrize("vocab", [4096, 50272])
def test_select_of_equal_values_over_all_beams(vocab):
    """Every continuation of every beam is worth the same: the lowest beam's lowest words."""
    for beams, n_best in ((16, 32), (5, 32), (16, 16)):
        x = np.full((beams, vocab), 0.5, np.float32)
        _check_select(x, np.full(beams, -3.0, np.float32), beams, n_best)
        _check_select(x, np.full(beams, -3.0, np.float32), beams, n_best, np.ones(beams, np.int32), eos=7)


def test_reorder_with_the_largest_range_of_pages():
    """A group that owns 2^20 pages: their bits fill most of a workgroup's memory.  The free ones are the last."""
    nh, dh, per, beams = 1, 64, 1 << 20, 3
    cfg = B.Cfg(nh * dh, nh, 64, 64, 64)
    pages = B.KVPages(cfg, per, int8=True, zero=False)
    stride = (per - 2) // beams
    table = np.full((beams, stride + 1), -1, np.int32)
    table[:, :stride] = np.arange(beams * stride).reshape(beams, stride)        # all but the last few pages are held
    pos = np.array([64 * stride, 64 * stride - 10, 64 * stride], np.int32)
    for t in (pages.k_codes, pages.v_codes):
        t[2 * stride - 1].random_(-127, 128)
    pages.k_meta[2 * stride - 1] = 0.5
    parents = np.array([0, 1, 1], np.int32)
    want = F.reorder(table, pos, parents, beams, per)
    got = B.fg_beam_reorder_paged(cfg, [pages], dev(table), dev(pos), dev(parents), beams, per)
    for a, b in zip(got, want[:3]):
        assert np.array_equal(host(a), b)
    (_, src, dst, n), = want[3]
    assert n == 64 and torch.equal(pages.k_codes[src], pages.k_codes[dst]) and torch.equal(pages.v_codes[src], pages.v_codes[dst])
    assert float(pages.k_meta[dst, 0]) == 0.5


def test_select_of_the_most_rows():
    rows, vocab = 65535, 12
    x = (np.random.default_rng(1).standard_normal((rows, vocab)) * 2).astype(np.float32)
    _check_select(x, np.zeros(rows, np.float32), 3, 4)
    with pytest.raises(B.FgError):
        B.fg_beam_select(B.Cfg(64, 1, 64, vocab, 64), torch.zeros((65536, vocab), device="cuda"), torch.zeros(65536, device="cuda"), 4)


def test_select_of_a_large_vocabulary():
    vocab = 3000001
    x = (np.random.default_rng(2).standard_normal((4, vocab)) * 2).astype(np.float32)
    x[1, -3:] += 30
    x[2, :2] += 30
    _check_select(x, np.array([-1, -2, -3, -1.5], np.float32), 4, 32)
