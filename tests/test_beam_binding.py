"""What the binding of beam search refuses before anything is launched: the tensors here are host ones, the refusals come first."""
import pytest
import torch

from paper_2303_06865_amd import binding as B

VOCAB = 1000


def _select(logits, rows, beams=4, **kw):
    return B.fg_beam_select(B.Cfg(64, 1, 64, VOCAB, 64), logits, torch.zeros(rows), beams, **kw)


@pytest.mark.parametrize("rows", [2, 4, 8])
def test_select_refuses_rows_that_overlap(rows):
    """One row that stands for several (a prompt's logits handed to all its beams as a view), and rows less than a vocabulary
    apart: a row distance of `vocab` in their place would read past their end."""
    one = torch.zeros(1, VOCAB)
    with pytest.raises(AssertionError, match="vocab elements apart"):
        _select(one.expand(rows, -1), rows, 2)
    with pytest.raises(AssertionError, match="vocab elements apart"):
        _select(torch.zeros(VOCAB + 16 * rows).as_strided((rows, VOCAB), (16, 1)), rows, 2)
    with pytest.raises(AssertionError, match="vocab elements apart"):
        _select(torch.zeros(rows * VOCAB).as_strided((rows, VOCAB), (VOCAB - 1, 1)), rows, 2)


def test_a_single_row_has_no_distance():
    """Whatever stride a view of one row has, it is the row: what is refused then is the host's memory."""
    for view in (torch.zeros(1, VOCAB), torch.zeros(VOCAB).as_strided((1, VOCAB), (0, 1)), torch.zeros(VOCAB).as_strided((1, VOCAB), (7, 1))):
        with pytest.raises(Exception) as e:
            _select(view, 1, 1)
        assert "vocab elements apart" not in str(e.value)
