"""Attention over 8-bit pages where elements of a query differ by many orders of magnitude, where a page's scale is an infinity,
and where few sequences of any length lie in long tables (split over workgroups), against binary64.

Tolerance.  Codes and queries enter the products exactly, as integer sums per digit of the query; the score is f times the sum of
four such numbers (f: the query's and the page's scales).  The digits of a number have magnitudes that add up to at most 3.02 times
its own (worst: a digit 1 over a digit -128 of 256).  So with A = sum |q_d k_d| scale, in units of 2^-24: the conversions and the four
products are off by 2 * 3.02 A, the two additions by 2 * 3.02 A, and f by 6 roundings of its own, of the score s.  The exponential and what follows
of it are off by 2^-21 as in test_gpu_i8_pages.  A relative error e of every weight moves a mean of values by at most 2 e max|v|; the
result is rounded to FP16 (2^-11 of it, 2^-25 below the normal numbers)."""
import numpy as np
import pytest
import torch

from paper_2303_06865_amd import binding as B
from paper_2303_06865_amd import synth
from tests import plain_i8 as P
from tests.test_gpu_i8_pages import _cfg, _rows, _table, _upload
from tests.util import assert_close, dev, host

pytestmark = pytest.mark.gpu


def _exact(plain, table, q, lens, nh, nkv, dh):
    """(outputs, tolerances) [b, nh, dh] in binary64."""
    outs, tols = [], []
    for i, n in enumerate(lens):
        x = q[i, :nh * dh].astype(np.float64).reshape(nkv, nh // nkv, dh)
        if n == 0:
            outs.append(np.zeros((nh, dh)))
            tols.append(np.zeros((nh, dh)))
            continue
        k, v = plain.rows(table, i, n)
        s = np.matmul(x, k.transpose(0, 2, 1)) / np.sqrt(dh)
        a = np.matmul(np.abs(x), np.abs(k).transpose(0, 2, 1)) / np.sqrt(dh)
        w = np.exp(s - s.max(-1, keepdims=True))
        o = np.matmul(w, v) / w.sum(-1, keepdims=True)
        e = 2.0 ** -24 * (4 * 3.02 * a + 6 * np.abs(s)).max(-1, keepdims=True) + 2.0 ** -21
        outs.append(o.reshape(nh, dh))
        tols.append((np.abs(o) * 2.0 ** -11 + 2.0 ** -25 + 2 * e * np.abs(v).max((1, 2))[:, None, None]).reshape(nh, dh))
    return np.stack(outs), np.stack(tols)


def _run(cfg, nh, nkv, dh, beams, q, table, lens, pages, **kw):
    seqs = B.Ragged(dev(table), None, dev(np.array(lens, np.int32)))
    return host(B.fg_decode_attention_beams_paged(cfg, nkv, beams, dev(q), q.shape[1], len(lens), pages, seqs, **kw)).reshape(-1, nh, dh)


def _close(got, want, tol):
    err = np.abs(got.astype(np.float64) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-30)).max())


@pytest.mark.parametrize("nh,nkv,dh,beams,b,n", [(2, 2, 128, 1, 2, 100), (2, 2, 64, 2, 4, 3000), (4, 1, 128, 1, 1, 3000), (6, 1, 64, 4, 4, 200),
                                                 (2, 2, 128, 4, 4, 70), (1, 1, 128, 1, 1100, 70), (1, 1, 64, 1, 2100, 70)])
@pytest.mark.parametrize("top", [1.0, 63.0, 70.0, 200.0, 2000.0, 60000.0])
def test_queries_with_one_large_element(nh, nkv, dh, beams, b, n, top):
    """The large element meets keys of zero; the scores are those of the others, down to subnormal ones."""
    lens = [n] * b
    stride = -(-n // 64)
    shared = min(b, 8)
    plain = P.I8Pages(shared * stride, nkv, dh, seed=int(top))
    table = np.tile(_table(shared, stride, plain.n, 1), (-(-b // shared), 1))[:b]
    table = np.repeat(table[::beams], beams, 0)
    r = np.random.default_rng(b)
    at = r.integers(0, dh)
    plain.codes[0][:, :, :, at] = 0
    plain.scales[0] *= 40
    plain.scales[1][:] = 2.0 ** -6
    q = _rows((b, nh * dh), 3)
    x = q.reshape(b, nh, dh)
    x[:, :, ::3] *= np.float16(2.0 ** -7)
    x[:, :, 1::5] *= np.float16(2.0 ** -14)
    x[:, :, at] = top
    x[::2, :, at] *= -1
    got = _run(_cfg(nh, dh), nh, nkv, dh, beams, q, table, lens, _upload(plain, B.Cfg(nkv * dh, nkv, 64, 64, 64)))
    some = sorted(set(range(min(b, 9))) | {b - 1})
    _close(got[some], *_exact(plain, table[some], q[some], [n] * len(some), nh, nkv, dh))


@pytest.mark.parametrize("dh", [64, 128])
def test_queries_of_any_magnitude(dh):
    """All elements of one size, from the smallest subnormal number to the largest number."""
    nh, n, b = 2, 90, 12
    plain = P.I8Pages(2 * b, nh, dh, seed=dh)
    table = _table(b, 2, plain.n, 1)
    q = np.random.default_rng(5).choice(np.array([-1.0, -0.75, 0.5, 1.0]), (b, nh * dh))
    q = (q * np.array([2.0 ** -24, 2.0 ** -23, 2.0 ** -16, 2.0 ** -8, 0.3, 1.99, 31.9, 63.97, 64, 127.9, 128, 60000])[:, None]).astype(np.float16)
    for i in range(b):   # the scores stay where the weights are ordinary
        plain.scales[0][table[i]] *= np.float32(2.0 / max(1.0, float(np.abs(q[i]).max())))
    got = _run(_cfg(nh, dh), nh, nh, dh, 1, q, table, [n] * b, _upload(plain, _cfg(nh, dh)))
    _close(got, *_exact(plain, table, q, [n] * b, nh, nh, dh))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("b,beams,pages,step", [(1, 1, 12, 4), (2, 2, 12, 4), (1, 1, 40, 4), (1100, 1, 5, 2), (2200, 2, 5, 2), (2100, 1, 3, 1),
                                                (2, 1, 3, 1)])
@pytest.mark.parametrize("behind", [False, True])
def test_an_infinite_scale_whatever_the_weights(dh, b, beams, pages, step, behind):
    """One page of the row has all the weight (the others' underflows).  A page of the row with a scale of infinity or NaN gives NaN
    or infinities also if its weight is nothing, whether it comes before or behind the one that counts (`step`: the wave that takes one
    takes the other)."""
    nh, n = 1, 64 * pages - 10
    heavy, place = (0, step) if behind else (step, 0)
    plain = P.I8Pages(pages + 1, nh, dh, seed=step)
    table = np.tile(np.random.default_rng(1).permutation(pages)[None], (b, 1)).astype(np.int32)
    if beams > 1:
        table[1::beams, place] = pages                      # row 0's own page is not row 1's
    q = np.ones((b, nh * dh), np.float16)
    plain.codes[0][:] = -100
    plain.scales[0][:] = 0.1
    plain.codes[0][table[0, heavy]] = 100
    cfg = _cfg(nh, dh)
    dev_pages = _upload(plain, cfg)
    good = _run(cfg, nh, nh, dh, beams, q, table, [n] * b, dev_pages)
    assert np.isfinite(good).all()
    for scales in (dev_pages.k_meta, dev_pages.v_meta):
        for value in (np.inf, np.nan):
            was = float(scales[int(table[0, place]), 0])
            scales[int(table[0, place]), 0] = value
            got = _run(cfg, nh, nh, dh, beams, q, table, [n] * b, dev_pages)
            scales[int(table[0, place]), 0] = was
            assert not np.isfinite(got[0]).any()
            if beams > 1:
                assert np.array_equal(got[1], good[1])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("sign", [-1, 1])
def test_an_infinite_key_scale_over_a_single_row(dh, sign):
    """The page's one key meets the query with products of one sign, at every order of magnitude: NaN nevertheless."""
    cfg = _cfg(1, dh)
    plain = P.I8Pages(2, 1, dh, seed=1)
    plain.codes[0][1] = sign
    plain.scales[0][1] = np.inf
    q = np.tile(np.array([33, 33 / 2 ** 8, 33 / 2 ** 16, 33 / 2 ** 24]), dh // 4)[None].astype(np.float16)
    for lens in ([65], [100]):
        got = _run(cfg, 1, 1, dh, 1, q, np.array([[0, 1]], np.int32), lens, _upload(plain, cfg))
        assert np.isnan(got).all()


@pytest.mark.parametrize("nh,nkv,dh", [(2, 2, 64), (2, 2, 128), (8, 2, 128), (6, 1, 64)])
@pytest.mark.parametrize("beams", [1, 2, 4])
def test_few_sequences_of_any_length_in_long_tables(nh, nkv, dh, beams):
    """Sequences are split over workgroups by what the table could hold: some splits find no page, some rows have none."""
    lens = [0, 1, 65, 4096][:max(4, beams)]
    b, stride = len(lens), 64
    plain = P.I8Pages(80, nkv, dh, seed=beams)
    r = np.random.default_rng(nh)
    table = np.stack([r.permutation(plain.n)[:stride] for _ in range(b)]).astype(np.int32)
    for i in range(b):
        table[i, :20] = table[i // beams * beams, :20]
    q = _rows((b, nh * dh), 4)
    cfg = _cfg(nh, dh)
    pages = _upload(plain, B.Cfg(nkv * dh, nkv, 64, 64, 64))
    assert B.decode_attention_beams_workspace(cfg, nkv, beams, b, stride).numel() > 4096      # there are splits
    for order in (lens, lens[::-1], [4096, 0, 300, 0]):
        got = _run(cfg, nh, nkv, dh, beams, q, table, order, pages)
        _close(got, *_exact(plain, table, q, order, nh, nkv, dh))


@pytest.mark.parametrize("beams", [1, 3])
def test_layer_splits_in_its_own_workspace(beams):
    """A layer on 8-bit pages in a long table is the same layer in one that is just long enough, where nothing is split (up to the
    order of sums)."""
    sh = synth.Shape(h1=256, nh=4, h2=2048, vocab=500, max_pos=8192, l=1)
    cfg = B.Cfg(sh.h1, sh.nh, sh.h2, sh.vocab, sh.max_pos)
    w = B.LayerWeights.from_numpy(synth.layer_tensors(sh, 0, 0, std=0.08, biases=True, random_ln=True), True)
    for pos in ([1000, 3, 0], [1400, 63, 1407]):
        b, plain = 3, P.I8Pages(3 * 22 + 1, 4, 64, seed=1)
        table = _table(b, 22, plain.n, 2)
        outs = []
        for stride in (22, 512):
            wide = np.full((b, stride), -1, np.int32)
            wide[:, :22] = table
            x = dev(_rows((b, sh.h1), 9))
            outs.append(host(B.fg_decode_layer_paged(cfg, w, x, _upload(plain, cfg), B.Ragged(dev(wide), None, dev(np.array(pos, np.int32))),
                                                     beams=beams)))
        assert np.isfinite(outs[0]).all()
        assert_close(outs[1], outs[0], "layer")
