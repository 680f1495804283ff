"""The plain form of reordering rows of any lengths, on the CPU: worked cases, and what it promises."""
import numpy as np
import pytest

from tests import plain_forks as F
from tests import plain_i8 as P


def _run(table, pos, parents, beams, per):
    return F.reorder(np.array(table, np.int32), np.array(pos, np.int32), np.array(parents, np.int32), beams, per)


def test_pins_of_a_page_held_as_a_full_one():
    """Page 1 is row 0's full page and row 1's begun one (or the other way round): row 1 gets a copy, row 0 a free page."""
    new, pos, missing, copies = _run([[0, 1, -1], [0, 1, -1]], [128, 70], [0, 1], 2, 6)
    assert new.tolist() == [[0, 1, 2], [0, 3, -1]] and copies == [(1, 1, 3, 16)] and not missing[0]
    new, pos, missing, copies = _run([[0, 1, -1], [0, 1, -1]], [70, 128], [0, 1], 2, 6)
    assert new.tolist() == [[0, 2, -1], [0, 1, 3]] and copies == [(0, 1, 2, 16)] and not missing[0]
    new, pos, missing, copies = _run([[0, 1, -1], [0, 1, 2]], [100, 130], [1, 0], 2, 6)       # after the parents are taken
    assert new.tolist() == [[0, 1, 2], [0, 3, -1]] and copies == [(1, 1, 3, 48)]
    new, pos, missing, copies = _run([[0, 1], [0, 1]], [128, 70], [0, 1], 2, 2)                # no page left, and a full table
    assert new.tolist() == [[0, 1], [0, -1]] and not copies and missing[0] == 2


@pytest.mark.parametrize("seed", range(40))
def test_the_next_position_is_the_row_s_alone(seed):
    r = np.random.default_rng(seed)
    beams, groups, stride = int(r.integers(1, 17)), int(r.integers(1, 4)), int(r.integers(2, 9))
    per = beams * stride + int(r.integers(0, beams + 1))
    table, pos = F.tree(r, groups, beams, stride, per)
    parents = r.integers(-1, beams + 1, groups * beams).astype(np.int32)
    new, npos, missing, copies = F.reorder(table, pos, parents, beams, per)
    copied = {i: (src, n) for i, src, _, n in copies}
    to = [dst for _, _, dst, _ in copies]
    assert len(set(to)) == len(to) and not set(to) & {src for _, src, _, _ in copies}
    for i in range(groups * beams):
        p = parents[i] if 0 <= parents[i] < beams else i % beams
        k = i // beams * beams + p
        n, at = int(npos[i]), int(npos[i]) // 64
        assert npos[i] == pos[k] and (new[i, :at] == table[k, :at]).all() and (new[i, at + 1:] == -1).all()
        if n % 64:
            src = copied[i][0] if i in copied else new[i, at]
            assert new[i, at] < 0 or (src == table[k, at] and (i not in copied or copied[i][1] >= n % 64))
        if new[i, at] >= 0:
            assert (new == new[i, at]).sum() == 1 and i // beams * per <= new[i, at] < (i // beams + 1) * per


def test_rows_of_equal_lengths_are_as_before():
    for seed in range(30):
        r = np.random.default_rng(seed)
        beams, stride = int(r.integers(1, 9)), int(r.integers(2, 6))
        per = beams * stride + beams
        table, _ = F.tree(r, 2, beams, stride, per)
        at = int(r.integers(0, 64 * stride - 64))
        pos = np.full(2 * beams, at, np.int32)
        for i in range(2 * beams):
            table[i, :at // 64 + 1] = table[i // beams * beams, :at // 64 + 1]
        parents = r.integers(0, beams, 2 * beams).astype(np.int32)
        for a, b in zip(F.reorder(table, pos, parents, beams, per), P.reorder(table, pos, parents, beams, per)):
            assert np.array_equal(a, b)
