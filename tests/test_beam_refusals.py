"""Arguments that the calls on 8-bit pages and of beam search refuse, on the host; and the plain forms' own pins."""
import ctypes as C

import numpy as np
import pytest

from paper_2303_06865_amd import binding as B
from tests import plain_i8 as P

A = 4096   # a fake, aligned address that is never dereferenced


def _cfg(h1=768, nh=12, vocab=50272):
    return B.fg_model_cfg(h1, nh, 4 * h1, vocab, 2048, 1e-5)


def _i8(n=64, km=A, vc=A, dtype=B.FG_I8P64):
    return B.fg_kv_pages(A, km, vc, A, dtype, n)


def test_append_and_attention_take_8_bit_pages_and_refuse_bad_ones():
    L, cfg = B.lib(), _cfg()
    seqs = B.fg_ragged(A, None, A, 2, 4)
    app = lambda pg, b=0, s=1, k=A: L.fg_kv_append_paged(C.byref(cfg), k, A, 2304, b, s, C.byref(pg), C.byref(seqs), None)  # noqa: E731
    assert app(_i8()) == B.FG_OK
    assert app(_i8(km=None)) == B.FG_ERR_NULL
    assert app(_i8(km=A + 2)) == B.FG_ERR_SHAPE
    assert app(_i8(km=A + 4)) == B.FG_OK             # scales are single numbers
    assert app(_i8(vc=A + 8)) == B.FG_ERR_SHAPE
    assert app(_i8(), b=1, k=A + 2) == B.FG_ERR_SHAPE
    att = L.fg_decode_attention_paged(C.byref(cfg), A, 2304, 0, C.byref(_i8()), C.byref(seqs), 1, A, None)
    assert att == B.FG_OK
    topk = L.fg_decode_attention_topk_paged(C.byref(cfg), A, 2304, 4, 3, C.byref(_i8()), C.byref(seqs), 1, A, None, None)
    assert topk == B.FG_ERR_UNSUPPORTED
    dense = B.fg_kv_cache(A, A, A, A, B.FG_I8P64, 4, 64, 0)
    assert L.fg_decode_attention(C.byref(cfg), A, 2304, 4, 3, C.byref(dense), 0, A, None) == B.FG_ERR_UNSUPPORTED
    assert L.fg_linear_workspace_bytes(C.byref(B.fg_mat(A, A, B.FG_I8P64, 0, 64, 64)), 0) == 0


def test_beam_attention_refusals():
    L, cfg, seqs = B.lib(), _cfg(), B.fg_ragged(A, None, A, 2, 4)

    def att(nkv=12, beams=2, b=4, pg=None, stride=2304, bias=0, q=A, ws=A, nws=1 << 40, seqs=seqs):
        return L.fg_decode_attention_beams_paged(C.byref(cfg), nkv, beams, q, stride, b, C.byref(pg or _i8()), C.byref(seqs), bias,
                                                 A, ws, nws, None)

    assert att(b=0) == B.FG_OK
    for bad in (dict(nkv=5), dict(nkv=0), dict(nkv=24), dict(beams=0), dict(beams=17, b=17), dict(beams=3), dict(b=-2), dict(stride=764),
                dict(stride=2305), dict(bias=-1), dict(q=A + 8)):
        assert att(**bad) == B.FG_ERR_SHAPE, bad
    assert att(pg=_i8(dtype=B.FG_Q4G64)) == B.FG_ERR_UNSUPPORTED
    assert att(pg=B.fg_kv_pages(A, None, A, None, B.FG_F16, 8)) == B.FG_ERR_UNSUPPORTED
    assert att(seqs=B.fg_ragged(A, None, None, 2, 4)) == B.FG_ERR_NULL
    assert att(q=None) == B.FG_ERR_NULL
    assert att(ws=None) == B.FG_ERR_WORKSPACE and att(nws=8) == B.FG_ERR_WORKSPACE
    size = lambda nkv=12, beams=2, b=4, stride=2: L.fg_decode_attention_beams_workspace_bytes(C.byref(cfg), nkv, beams, b, stride)  # noqa: E731
    assert size() > 0 and size(nkv=5) == 0 and size(beams=3) == 0 and size(stride=0) == 0 and size(b=0) == 0


def test_gather_refusals():
    L, cfg, seqs = B.lib(), _cfg(), B.fg_ragged(A, None, None, 2, 4)
    ga = lambda b=1, s=1, k=A, v=A, stride=768, pg=None: L.fg_kv_gather_paged(C.byref(cfg), C.byref(pg or _i8()), C.byref(seqs), b, s, k, v,  # noqa: E731
                                                                             stride, None)
    assert ga(b=0) == B.FG_OK and ga(s=0) == B.FG_OK
    assert ga(b=-1) == B.FG_ERR_SHAPE and ga(s=-1) == B.FG_ERR_SHAPE
    assert ga(stride=760) == B.FG_ERR_SHAPE and ga(stride=769) == B.FG_ERR_SHAPE
    assert ga(k=None) == B.FG_ERR_NULL and ga(v=None) == B.FG_ERR_NULL and ga(k=A + 8) == B.FG_ERR_SHAPE
    assert ga(pg=_i8(dtype=7)) == B.FG_ERR_UNSUPPORTED


def test_select_refusals():
    L = B.lib()

    def sel(n=2, beams=4, best=4, stride=50272, done=None, eos=-1, logits=A, scores=A, out=A, ws=A, nws=1 << 40, cfg=_cfg()):
        return L.fg_beam_select(C.byref(cfg), n, beams, best, logits, stride, scores, done, eos, out, A, A, None, ws, nws, None)

    assert sel(n=0) == B.FG_OK
    for bad in (dict(n=-1), dict(beams=0), dict(beams=17), dict(best=0), dict(best=33), dict(stride=50271), dict(eos=50272), dict(done=A),
                dict(n=1 << 30)):
        assert sel(**bad) == B.FG_ERR_SHAPE, bad
    for bad in (dict(logits=None), dict(scores=None), dict(out=None)):
        assert sel(**bad) == B.FG_ERR_NULL, bad
    assert sel(ws=None) == B.FG_ERR_WORKSPACE and sel(nws=16) == B.FG_ERR_WORKSPACE and sel(ws=A + 8) == B.FG_ERR_SHAPE
    size = lambda n=2, beams=4, best=4: L.fg_beam_select_workspace_bytes(C.byref(_cfg()), n, beams, best)  # noqa: E731
    assert size() > 0 and size(n=0) == 0 and size(beams=17) == 0 and size(best=33) == 0


def test_reorder_refusals():
    L, cfg = B.lib(), _cfg()

    def reo(l=2, n=2, beams=4, per=8, pages=None, stride=4, parents=A, tin=A, pin=A, tout=A, pout=A, ws=A, nws=1 << 40):  # noqa: E741
        pages = pages or [_i8(16), _i8(16)]
        arr = (B.fg_kv_pages * len(pages))(*pages)
        return L.fg_beam_reorder_paged(C.byref(cfg), l, arr, n, beams, per, parents, tin, pin, stride, tout, pout, None, ws, nws, None)

    assert reo(n=0) == B.FG_OK
    for bad in (dict(l=0), dict(n=-1), dict(beams=0), dict(beams=17), dict(per=0), dict(per=9), dict(stride=0), dict(stride=1 << 26),
                dict(pages=[_i8(16), _i8(17)])):
        assert reo(**bad) == B.FG_ERR_SHAPE, bad
    assert reo(pages=[_i8(16), _i8(16, dtype=B.FG_Q4G64)]) == B.FG_ERR_UNSUPPORTED
    assert reo(pages=[_i8(16, dtype=7)], l=1) == B.FG_ERR_UNSUPPORTED
    assert reo(pages=[_i8(1 << 30)], l=1, n=1, per=(1 << 20) + 1) == B.FG_ERR_UNSUPPORTED
    for bad in (dict(parents=None), dict(tin=None), dict(pin=None), dict(tout=None), dict(pout=None), dict(pages=[_i8(16, km=None)], l=1)):
        assert reo(**bad) == B.FG_ERR_NULL, bad
    assert reo(ws=None) == B.FG_ERR_WORKSPACE and reo(nws=16) == B.FG_ERR_WORKSPACE
    assert L.fg_beam_reorder_workspace_bytes(2, 4) > 0 and L.fg_beam_reorder_workspace_bytes(0, 4) == 0


@pytest.mark.parametrize("dh", [64, 128])
def test_plain_pages_hold_rows_within_half_a_step(dh):
    """What the format promises, on the plain form itself: half a scale when stored at once; every growth adds at most half
    of the scale then, and the scales of a page only grow, so a row is off by at most (1 + growths) / 2 of the last one.  The
    number that is rounded to a code comes of two binary32 roundings (the reciprocal or ratio, the product): of at most 127, it
    is off by 127 * 2^-23 steps, which is 2^-15 of half a step."""
    r = np.random.default_rng(dh)
    pages, table = P.I8Pages(2, 2, dh), np.array([[1, 0]])
    k, v = (r.standard_normal((100, 2 * dh)).astype(np.float16) for _ in range(2))
    pages.append(table, 0, 0, k[:70], v[:70])
    growths = np.zeros((2, 2, 2))
    for p in range(70, 100):
        before = [s.copy() for s in pages.scales]
        pages.append(table, 0, p, k[p:p + 1], v[p:p + 1])
        growths += np.stack(pages.scales) > np.stack(before)
    assert growths[:, 0].max() >= 1 and not growths[:, 1].any()
    for t, (x, got) in enumerate(zip((k, v), pages.rows(table, 0, 100))):
        err = np.abs(got - x.reshape(100, 2, dh).transpose(1, 0, 2).astype(np.float64)).max(-1)      # [nh, 100]
        for page, sl in ((1, slice(0, 64)), (0, slice(64, 100))):
            bound = pages.scales[t][page] * (1 + growths[t][page]) / 2 * (1 + 2.0 ** -15)
            assert (err[:, sl] <= bound[:, None]).all()


def test_plain_select_pins():
    """Two beams worked by hand: equal logits tie to the lower word, equal values to the lower beam."""
    x = np.log(np.array([[1.0, 2.0, 2.0, 3.0], [1.0, 2.0, 2.0, 3.0]])).astype(np.float32)
    got = P.select(x, np.array([0.0, 0.0], np.float32), 2, 5)[0]
    assert [(j, w) for j, w, _, _ in got] == [(0, 3), (1, 3), (0, 1), (0, 2), (1, 1)]
    assert abs(got[0][2] - np.log(3 / 8)) < 1e-6
    got = P.select(x, np.array([-np.inf, 0.0], np.float32), 2, 5)[0]
    assert [(j, w) for j, w, _, _ in got] == [(1, 3), (1, 1), (1, 2), (1, 0), (-1, -1)]
    got = P.select(x, np.array([-0.5, 0.0], np.float32), 2, 2, done=np.array([1, 0]), eos=0)[0]
    assert got[0][:2] == (0, 0) and got[0][3] == 1 and got[1][:2] == (1, 3) and got[1][3] == 0


def test_plain_reorder_pins():
    """Two beams, 70 rows cached (page 0 shared, pages 1 and 2 begun), both continue beam 1: the first keeps page 2, the
    second takes the lowest page that nobody holds, which is page 1."""
    table = np.array([[0, 1, -1], [0, 2, -1]], np.int32)
    new, pos, missing, copies = P.reorder(table, np.array([70, 70], np.int32), np.array([1, 1]), 2, 4)
    assert new.tolist() == [[0, 2, -1], [0, 1, -1]] and pos.tolist() == [70, 70] and copies == [(1, 2, 1, 16)] and missing[0] == 0
    new, _, missing, copies = P.reorder(table, np.array([128, 128], np.int32), np.array([1, 0]), 2, 4)
    assert new.tolist() == [[0, 2, 3], [0, 1, -1]] and missing[0] == 1 and not copies
