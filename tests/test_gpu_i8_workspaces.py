"""One scratch buffer, made for the largest batch, in calls whose batches shrink as sequences finish: the bits are those of calls
with scratch of their own."""
import numpy as np
import pytest

from paper_2303_06865_amd import binding as B
from tests import plain_i8 as P
from tests.test_gpu_i8_pages import _cfg, _rows, _upload
from tests.util import dev, host

pytestmark = pytest.mark.gpu


def test_attention_of_shrinking_batches():
    nh, dh, beams, stride = 32, 128, 2, 64
    cfg, b = _cfg(nh, dh), 16
    plain = P.I8Pages(70, nh, dh, seed=1)
    pages = _upload(plain, cfg)
    table = np.stack([np.random.default_rng(i).permutation(plain.n)[:stride] for i in range(b)]).astype(np.int32)
    pos = np.random.default_rng(0).integers(1, 64 * stride, b).astype(np.int32)
    q = _rows((b, nh * dh), 3)
    ws = B.decode_attention_beams_workspace(cfg, nh, beams, b, stride)
    ws.fill_(255)                                       # NaN, if anybody read it before writing it
    for n in (16, 14, 8, 6, 4, 2):
        seqs = B.Ragged(dev(table[:n]), None, dev(pos[:n]))
        got, want = (host(B.fg_decode_attention_beams_paged(cfg, nh, beams, dev(q[:n]), nh * dh, n, pages, seqs, ws=w)) for w in (ws, None))
        assert np.isfinite(got).all() and np.array_equal(got, want)


def test_selection_of_shrinking_batches():
    beams, vocab = 4, 50272
    cfg = B.Cfg(64, 1, 64, vocab, 64)
    x = (np.random.default_rng(1).standard_normal((20 * beams, vocab)) * 2).astype(np.float32)
    scores = np.linspace(-9, -1, 20 * beams).astype(np.float32)
    ws = B.beam_select_workspace(cfg, 20, beams, 8)
    ws.fill_(255)
    for n, best in ((20, 8), (19, 8), (18, 8), (18, 4), (7, 8), (1, 1)):
        got, want = ([host(t) for t in B.fg_beam_select(cfg, dev(x[:n * beams]), dev(scores[:n * beams]), beams, best, ws=w)] for w in (ws, None))
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
