"""8-bit cache pages on the GPU: storing (bit for bit), reading back (bit for bit), attention against binary64.

Tolerance of attention.  The result is rounded to FP16: 2^-11 of its size (2^-25 below the normal numbers).  Before that, a score
of size s is off by a few binary32 roundings of its terms and of itself, at most 8 * 2^-24 * s with s the largest score (sums of
128 products of which most are smaller), its exponential by as much relatively, and 2^-22 from the exponential itself; weights
are kept to 2^-24 or better.  An output is a weighted mean of values, so it is off by at most twice the largest relative error
of a weight times the largest value: 2 (8 * 2^-24 * max(s, 1) + 2^-21) max|v|."""
import numpy as np
import pytest
import torch

from paper_2303_06865_amd import binding as B
from tests import plain_i8 as P
from tests.util import dev, host

pytestmark = pytest.mark.gpu


def _cfg(nh, dh):
    return B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 1 << 20)


def _upload(plain, cfg):
    pages = B.KVPages(cfg, plain.n, int8=True)
    kc, vc = plain.device_codes()
    for t, a in ((pages.k_codes, kc), (pages.v_codes, vc), (pages.k_meta, plain.scales[0]), (pages.v_meta, plain.scales[1])):
        t.copy_(dev(a))
    return pages


def _same(pages, plain):
    kc, vc = plain.device_codes()
    assert np.array_equal(host(pages.k_meta).view(np.uint32), plain.scales[0].view(np.uint32))
    assert np.array_equal(host(pages.v_meta).view(np.uint32), plain.scales[1].view(np.uint32))
    assert np.array_equal(host(pages.k_codes), kc)
    assert np.array_equal(host(pages.v_codes), vc)


def _rows(shape, seed, std=1.0):
    return (np.random.default_rng(seed).standard_normal(shape) * std).astype(np.float16)


def _table(n_seqs, stride, n_pages, seed):
    return np.random.default_rng(seed).permutation(n_pages)[:n_seqs * stride].reshape(n_seqs, stride).astype(np.int32)


@pytest.mark.parametrize("nh,dh", [(1, 128), (3, 128), (5, 64), (12, 64)])
@pytest.mark.parametrize("s,pos", [(1, [0, 1, 15, 16, 63]), (1, [64, 65, 127, 190, 5]), (3, [62, 0, 13, 126, 61]), (64, [0, 0, 64, 0, 64]),
                                   (70, [0, 10, 58, 63, 1]), (150, [0, 1, 63, 64, 33])])
def test_append_bit_for_bit(nh, dh, s, pos):
    b, cfg = len(pos), _cfg(nh, dh)
    plain = P.I8Pages(5 * b + 3, nh, dh, seed=s)
    table = _table(b, 5, plain.n, 3)
    table[1, 4] = -1          # no page there: dropped
    table[2, 3] = plain.n     # nor there
    pages = _upload(plain, cfg)
    ids = np.array([4, 0, 3, 1, 2], np.int32)
    qkv = _rows((b * s, 3 * nh * dh), 7)
    qkv[0, nh * dh:] = 0
    if s == 1:
        qkv[3, nh * dh:] *= 4     # grows the page's scale
    for i in range(b):
        rows = qkv[i * s:(i + 1) * s]
        plain.append(table, int(ids[i]), pos[i], rows[:, nh * dh:2 * nh * dh], rows[:, 2 * nh * dh:])
    d = dev(qkv)
    seqs = B.Ragged(dev(table), dev(ids), dev(np.array(pos, np.int32)))
    B.fg_kv_append_paged(cfg, d[:, nh * dh:], d[:, 2 * nh * dh:], 3 * nh * dh, b, s, pages, seqs)
    _same(pages, plain)


@pytest.mark.parametrize("dh", [64, 128])
def test_append_row_by_row_grows_scales(dh):
    """A whole page one row at a time, magnitudes rising, falling and zero, and rows beyond it in the next page."""
    nh, cfg = 2, _cfg(2, dh)
    plain, table = P.I8Pages(3, nh, dh), np.array([[2, 0]], np.int32)
    pages, dt = _upload(plain, cfg), dev(table)
    for p in range(70):
        std = [0.0, 1e-3, 1.0, 0.5, 3.0, 100.0][p % 6] if p < 40 else 2.0 ** (p - 40)
        kv = np.clip(_rows((1, 2 * nh * dh), p).astype(np.float32) * std, -60000, 60000).astype(np.float16)
        plain.append(table, 0, p, kv[:, :nh * dh], kv[:, nh * dh:])
        d = dev(kv)
        B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, 1, 1, pages, B.Ragged(dt, None, dev(np.array([p], np.int32))))
    _same(pages, plain)


@pytest.mark.parametrize("s", [1, 5, 70])
def test_append_same_sequence_twice_in_one_call(s):
    """Rows of one sequence that one call names several times are stored in the order of the rows."""
    nh, dh, cfg = 3, 128, _cfg(3, 128)
    b = 70
    pos = (10 + s * (np.arange(b) // 2)).astype(np.int32)
    ids = (np.arange(b) % 2).astype(np.int32)
    stride = int(pos.max() + s) // 64 + 1
    plain = P.I8Pages(2 * stride, nh, dh)
    table = _table(2, stride, plain.n, 5)
    pages = _upload(plain, cfg)
    kv = _rows((b * s, 2 * nh * dh), 9)
    for i in range(b):
        plain.append(table, int(ids[i]), int(pos[i]), kv[i * s:(i + 1) * s, :nh * dh], kv[i * s:(i + 1) * s, nh * dh:])
    d = dev(kv)
    B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, b, s, pages, B.Ragged(dev(table), dev(ids), dev(pos)))
    _same(pages, plain)


def test_append_leaves_everything_else():
    """Bad ids and positions store nothing; rows behind the new ones in a page keep their values; other pages are untouched."""
    nh, dh, cfg = 2, 64, _cfg(2, 64)
    plain = P.I8Pages(6, nh, dh, seed=1)
    table = _table(3, 2, 6, 2)
    pages = _upload(plain, cfg)
    ids, pos = np.array([-1, 3, 0, 1, 2], np.int32), np.array([0, 0, -5, 128, 20], np.int32)
    kv = _rows((5, 2 * nh * dh), 3, std=0.1)
    plain.append(table, 2, 20, kv[4:, :nh * dh], kv[4:, nh * dh:])
    d = dev(kv)
    B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, 5, 1, pages, B.Ragged(dev(table), dev(ids), dev(pos)))
    _same(pages, plain)


@pytest.mark.parametrize("nh,dh", [(3, 128), (5, 64)])
@pytest.mark.parametrize("s,at", [(1, 10), (1, 0), (70, 10)])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_append_of_infinities_and_nan(nh, dh, s, at, value):
    """The page and head that gets one is NaN as a whole, and stays so for rows stored behind it; all others are as without it.
    Storing the page's first position again makes it a page like any other."""
    cfg, h1 = _cfg(nh, dh), nh * dh
    good, odd = B.KVPages(cfg, 3, int8=True), B.KVPages(cfg, 3, int8=True)
    table = dev(np.array([[2, 0, 1]], np.int32))
    put = lambda p, k, v, pos: B.fg_kv_append_paged(cfg, dev(k), dev(v), h1, 1, k.shape[0], p, B.Ragged(table, None, dev(np.array([pos], np.int32))))
    first, rows, behind = _rows((2, 64, h1), 1), _rows((2, s, h1), 2, 3.0), _rows((2, 1, h1), 3)
    bad = rows.copy()
    bad[0, s - 1, dh + 3], bad[1, s - 1, dh + 9] = value, value      # head 1, the last row
    page = (at + s - 1) // 64
    for p, x in ((good, rows), (odd, bad)):
        if at:
            put(p, first[0, :at], first[1, :at], 0)
        put(p, x[0], x[1], at)
        put(p, behind[0], behind[1], at + s)
    n = at + s + 1
    read = lambda p: [host(t).reshape(n, nh, dh) for t in B.fg_kv_gather_paged(cfg, p, B.Ragged(table), 1, n)]
    for a, b in zip(read(good), read(odd)):
        assert np.isfinite(a).all()
        assert np.isnan(b[64 * page:, 1]).all()
        b[64 * page:, 1] = a[64 * page:, 1]
        assert np.array_equal(a, b)
    for p in (good, odd):
        put(p, first[0], first[1], 64 * page)
    for a, b in zip(read(good), read(odd)):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("fmt", ["i8", "f16", "q4", "q4h"])
@pytest.mark.parametrize("nh,dh,s", [(3, 128, 1), (5, 64, 77), (2, 128, 130), (8, 64, 64)])
def test_gather_reads_rows_back(fmt, nh, dh, s):
    cfg, b = _cfg(nh, dh), 4
    n_pages = 20
    table = _table(b, 4, n_pages, 1)
    table[3, 1] = -1
    pos, ids = np.array([0, 63, 100, 17], np.int32), np.array([2, 0, 3, 1], np.int32)
    r = np.random.default_rng(4)
    if fmt == "i8":
        plain = P.I8Pages(n_pages, nh, dh, seed=2)
        pages = _upload(plain, cfg)
        vals = [(plain.scales[t][:, :, None, None] * plain.codes[t].astype(np.float32)).astype(np.float16) for t in range(2)]
    elif fmt == "f16":
        pages = B.KVPages(cfg, n_pages, quantized=False)
        vals = [_rows((n_pages, nh, 64, dh), t) for t in range(2)]
        pages.k_codes.copy_(dev(vals[0]))
        pages.v_codes.copy_(dev(vals[1]))
    else:
        pages = B.KVPages(cfg, n_pages, meta_f16=fmt == "q4h")
        vals = []
        for codes, meta in ((pages.k_codes, pages.k_meta), (pages.v_codes, pages.v_meta)):
            c = r.integers(0, 256, tuple(codes.shape)).astype(np.uint8)
            m = np.stack((r.uniform(-3, -1, codes.shape[:3] + (dh // 64,)), r.uniform(0.1, 0.4, codes.shape[:3] + (dh // 64,))), -1)
            m = m.astype(np.float16 if fmt == "q4h" else np.float32)
            codes.copy_(dev(c))
            meta.copy_(dev(m))
            nib = np.stack((c & 15, c >> 4), -1).reshape(n_pages, nh, 64, dh // 64, 64).astype(np.float64)
            exact = nib * m[..., 1:].astype(np.float64) + m[..., :1].astype(np.float64)   # rounded to binary32, then to FP16
            vals.append(exact.astype(np.float32).astype(np.float16).reshape(n_pages, nh, 64, dh))
    wide = nh * dh + 24    # rows apart, and a guard between them
    out = torch.full((2, b, s, wide), 7.0, dtype=torch.float16, device="cuda")
    B.fg_kv_gather_paged(cfg, pages, B.Ragged(dev(table), dev(ids), dev(pos)), b, s, out[0], out[1], wide)
    got = host(out)
    assert (got[..., nh * dh:] == 7).all()
    for i in range(b):
        for j in range(s):
            p = pos[i] + j
            page = table[ids[i], p // 64] if p // 64 < 4 else -1
            for t in range(2):
                want = vals[t][page, :, p % 64].reshape(-1) if page >= 0 else np.zeros(nh * dh, np.float16)
                assert np.array_equal(got[t, i, j, :nh * dh], want), (i, j, t)
    k, v = B.fg_kv_gather_paged(cfg, pages, B.Ragged(dev(table)), b, s)     # from position 0, sequences in order
    assert np.array_equal(host(k)[0, 0], vals[0][table[0, 0], :, 0].reshape(-1)) and v.shape == (b, s, nh * dh)


def _attend_case(nh, nkv, dh, lens, beams, shared, seed, q_std=1.0, long_rows=None):
    """A pool and table where the rows of a group share the pages of their first `shared` rows (whole pages)."""
    b = len(lens)
    stride = max(1, -(-max(lens) // 64))
    plain = P.I8Pages(b * stride + 2, nkv, dh, seed=seed)
    table = _table(b, stride, plain.n, seed)
    for i in range(b):
        n = min(shared, lens[i], lens[i // beams * beams]) // 64
        table[i, :n] = table[i // beams * beams, :n]
    q = _rows((b, nh * dh + 2 * nkv * dh), seed + 1, q_std)
    return plain, table, q


def _check_attention(plain, table, q, lens, nh, nkv, dh, got, ids=None):
    for i, n in enumerate(lens):
        k, v = plain.rows(table, i if ids is None else int(ids[i]), n)
        want, smax = P.attention(q[i, :nh * dh].reshape(nh, dh), k, v, 1 / np.sqrt(dh))
        top = np.abs(v).max() if n else 0.0
        tol = np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + 2 * (8 * 2.0 ** -24 * max(smax, 1.0) + 2.0 ** -21) * top
        err = np.abs(got[i].astype(np.float64) - want)
        assert (err <= tol).all(), (i, n, float((err / np.maximum(tol, 1e-30)).max()))


@pytest.mark.parametrize("nh,nkv,dh", [(3, 3, 128), (12, 12, 64), (8, 2, 128), (6, 1, 64), (10, 2, 64), (32, 2, 128), (34, 2, 64)])
@pytest.mark.parametrize("beams", [1, 2, 4, 5])
def test_attention_against_64_bits(nh, nkv, dh, beams):
    lens = [1, 64, 63, 65, 130, 200, 17, 0, 128, 1, 700, 33, 255, 257, 90, 64, 5, 2, 300, 320][:4 * beams]
    plain, table, q = _attend_case(nh, nkv, dh, lens, beams, 128, seed=beams)
    cfg = _cfg(nh, dh)
    pages = _upload(plain, B.Cfg(nkv * dh, nkv, 4 * nkv * dh, 1000, 512))
    got = B.fg_decode_attention_beams_paged(cfg, nkv, beams, dev(q), q.shape[1], len(lens), pages,
                                            B.Ragged(dev(table), None, dev(np.array(lens, np.int32))))
    _check_attention(plain, table, q, lens, nh, nkv, dh, host(got))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("beams,b", [(1, 1), (4, 4), (1, 3), (16, 16), (3, 96)])
def test_attention_of_beams_with_a_long_prefix(dh, beams, b):
    """Equal lengths as in beam search; few rows (long sequences split over workgroups) and many."""
    nh = 4
    n = 3000 if b < 20 else 333
    lens = [n] * b
    plain, table, q = _attend_case(nh, nh, dh, lens, beams, n - 100, seed=b, q_std=2.0)
    cfg = _cfg(nh, dh)
    pages = _upload(plain, cfg)
    pos = dev(np.array(lens, np.int32) - 1)
    got = B.fg_decode_attention_beams_paged(cfg, nh, beams, dev(q), q.shape[1], b, pages, B.Ragged(dev(table), None, pos), rows_bias=1)
    _check_attention(plain, table, q, lens, nh, nh, dh, host(got))
    one = B.fg_decode_attention_paged(cfg, dev(q), q.shape[1], b, pages, B.Ragged(dev(table), None, pos), rows_bias=1)
    _check_attention(plain, table, q, lens, nh, nh, dh, host(one))


def test_attention_of_ids_and_bad_tables():
    """Rows name their sequences; entries out of range read some page of the pool, lengths stop at the table's end."""
    nh, dh, cfg = 2, 128, _cfg(2, 128)
    plain, table, q = _attend_case(nh, nh, dh, [100, 40, 128, 70], 1, 0, seed=9)
    pages = _upload(plain, cfg)
    ids = np.array([2, 0, 3, 1], np.int32)
    lens = [128, 100, 70, 40]
    seqs = B.Ragged(dev(table), dev(ids), dev(np.array(lens, np.int32)))
    got = host(B.fg_decode_attention_beams_paged(cfg, nh, 2, dev(q), q.shape[1], 4, pages, seqs))
    _check_attention(plain, table, q, lens, nh, nh, dh, got, ids)
    bad = table.copy()
    bad[0, 1], bad[1, 0] = plain.n + 5, -3
    fixed = np.clip(bad, 0, plain.n - 1)
    odd = np.array([1 << 30, 40, -7, 70], np.int32)
    got = host(B.fg_decode_attention_beams_paged(cfg, nh, 2, dev(q), q.shape[1], 4, pages, B.Ragged(dev(bad), None, dev(odd))))
    _check_attention(plain, fixed, q, [128, 40, 0, 70], nh, nh, dh, got)
    far = B.Ragged(dev(table), dev(np.array([9, -9, 1, 0], np.int32)), dev(np.array(lens, np.int32)))
    got = host(B.fg_decode_attention_beams_paged(cfg, nh, 1, dev(q), q.shape[1], 4, pages, far))
    _check_attention(plain, table, q, lens, nh, nh, dh, got, np.array([3, 0, 1, 0]))


@pytest.mark.parametrize("nh,nkv,b,beams,n,ws", [(1, 1, 2, 1, 17000, False), (1, 1, 132, 2, 16900, True), (1, 1, 1100, 1, 8700, True),
                                                 (16, 1, 260, 1, 4300, True), (2, 2, 40, 4, 16700, True)])
def test_attention_of_many_pages(nh, nkv, b, beams, n, ws):
    """More pages than a wave keeps at once, at every number of waves a unit.  All sequences name the same few hundred pages (the
    beams of a group differ in forty pages), so that some rows stand for all."""
    dh = 64
    stride = n // 64 + 1
    plain = P.I8Pages(stride + 40 * beams, nkv, dh, seed=n)
    r = np.random.default_rng(b)
    one = r.permutation(plain.n)
    table = np.empty((b, stride), np.int32)
    for j in range(beams):
        row = one[:stride].copy()
        row[20:60] = one[stride + 40 * j:stride + 40 * (j + 1)]
        table[j::beams] = row
    q = _rows((b, nh * dh), 5)
    cfg = _cfg(nh, dh)
    pages = _upload(plain, B.Cfg(nkv * dh, nkv, 64, 64, 64))
    seqs = B.Ragged(dev(table), None, dev(np.full(b, n, np.int32)))
    if ws:
        got = host(B.fg_decode_attention_beams_paged(cfg, nkv, beams, dev(q), nh * dh, b, pages, seqs))
    else:
        got = host(B.fg_decode_attention_paged(cfg, dev(q), nh * dh, b, pages, seqs))
    rows = sorted({0, 1 % b, b // 2, b - 1} | set(range(min(beams, b))))
    for i in rows:
        _check_attention(plain, table[i:i + 1], q[i:i + 1], [n], nh, nkv, dh, got[i:i + 1])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("nh,b,beams,stride", [(12, 16, 1, 100), (8, 64, 4, 150), (33, 32, 1, 40), (1, 4100, 1, 2), (1, 4100, 1, 5)])
def test_attention_with_room_for_much(nh, b, beams, stride, dh):
    """Tables that could hold more pages than a last-level cache, whose sequences are short (head size 64, 4100
    units with two pages: ones that it could keep): 1, 2 and 4 waves a unit."""
    lens = [(0, 1, 63, 64, 100, 128)[i % 6] for i in range(b)]
    plain = P.I8Pages(40, nh, dh, seed=stride)
    table = np.full((b, stride), -1, np.int32)
    r = np.random.default_rng(nh)
    for g in range(0, b, beams):
        table[g:g + beams, :2] = r.integers(0, plain.n, 2)
        table[g + beams - 1, 1] = r.integers(0, plain.n)
    q = _rows((b, nh * dh), 3)
    cfg = _cfg(nh, dh)
    pages = _upload(plain, cfg)
    seqs = B.Ragged(dev(table), None, dev(np.array(lens, np.int32)))
    got = host(B.fg_decode_attention_beams_paged(cfg, nh, beams, dev(q), nh * dh, b, pages, seqs))
    some = sorted(set(range(min(b, 12))) | {b // 2, b - 1})
    _check_attention(plain, table[some], q[some], [lens[i] for i in some], nh, nh, dh, got[some])


def test_pages_beyond_32_bits():
    """Codes whose offsets pass 2^32: stored, read back, copied and attended to."""
    nh, dh, cfg = 32, 128, _cfg(32, 128)
    n_pages = (1 << 32) // (nh * 64 * dh) + 40
    pages = B.KVPages(cfg, n_pages, int8=True, zero=False)
    table = np.array([[n_pages - 1, n_pages - 2]], np.int32)
    small = P.I8Pages(2, nh, dh)
    kv = _rows((100, 2 * nh * dh), 1)
    small.append(np.array([[0, 1]]), 0, 0, kv[:, :nh * dh], kv[:, nh * dh:])
    d = dev(kv)
    B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, 1, 100, pages, B.Ragged(dev(table)))
    k, v = B.fg_kv_gather_paged(cfg, pages, B.Ragged(dev(table)), 1, 100)
    want = small.rows(np.array([[0, 1]]), 0, 100)
    for got, x in zip((k, v), want):
        assert np.array_equal(host(got)[0], x.astype(np.float32).astype(np.float16).transpose(1, 0, 2).reshape(100, -1))
    two = dev(np.repeat(table, 2, 0))
    pos = dev(np.array([100, 100], np.int32))
    got_t, _, _ = B.fg_beam_reorder_paged(cfg, [pages], two, pos, dev(np.array([1, 0], np.int32)), 2, n_pages)
    assert host(got_t).tolist() == [[n_pages - 1, n_pages - 2], [n_pages - 1, 0]]
    q = _rows((2, nh * dh), 2)
    out = B.fg_decode_attention_beams_paged(cfg, nh, 2, dev(q), nh * dh, 2, pages, B.Ragged(got_t, None, pos))
    _check_attention(small, np.array([[0, 1], [0, 1]]), q, [100, 100], nh, nh, dh, host(out))


def test_rows_past_the_table():
    """Rows that run past the table's end are dropped when stored and read as zeros, also before position 0."""
    nh, dh, cfg = 2, 128, _cfg(2, 128)
    plain, table = P.I8Pages(5, nh, dh, seed=1), np.array([[4, 1]], np.int32)
    pages = _upload(plain, cfg)
    kv = _rows((70, 2 * nh * dh), 3)
    plain.append(table, 0, 100, kv[:, :nh * dh], kv[:, nh * dh:])
    d, at = dev(kv), lambda p: B.Ragged(dev(table), None, dev(np.array([p], np.int32)))
    B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, 1, 70, pages, at(100))
    _same(pages, plain)
    want = [x.astype(np.float32).astype(np.float16).transpose(1, 0, 2).reshape(128, -1) for x in plain.rows(table, 0, 128)]
    k, v = (host(t)[0] for t in B.fg_kv_gather_paged(cfg, pages, at(120), 1, 80))
    assert np.array_equal(k[:8], want[0][120:]) and np.array_equal(v[:8], want[1][120:]) and not k[8:].any() and not v[8:].any()
    k, v = (host(t)[0] for t in B.fg_kv_gather_paged(cfg, pages, at(-70), 1, 90))
    assert np.array_equal(k[70:], want[0][:20]) and np.array_equal(v[70:], want[1][:20]) and not k[:70].any() and not v[:70].any()


def test_attention_extremes():
    """A score that dwarfs the others, a query of zeros, scales of zero, a page whose rows behind the end hold anything."""
    nh, dh, cfg = 4, 128, _cfg(4, 128)
    lens = [500, 500, 500, 100]
    plain, table, q = _attend_case(nh, nh, dh, lens, 1, 0, seed=3, q_std=8.0)
    q[1] = 0
    q[2, 0:dh] *= np.float16(0.001)
    plain.scales[0][table[2, 3]] = 0
    plain.scales[1][table[2, 5]] = 0
    plain.codes[0][table[3, 1], :, 36:] = 127
    plain.codes[1][table[3, 1], :, 36:] = -127
    pages = _upload(plain, cfg)
    got = B.fg_decode_attention_paged(cfg, dev(q), q.shape[1], 4, pages, B.Ragged(dev(table), None, dev(np.array(lens, np.int32))))
    _check_attention(plain, table, q, lens, nh, nh, dh, host(got))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("b,beams,n", [(4, 4, 100), (4, 1, 100), (4, 2, 3000), (1200, 2, 70)])
def test_attention_keeps_infinities_to_whom_they_belong(dh, b, beams, n):
    """A query with an infinity or a NaN gives NaN; a page whose scale is one gives NaN to the beams that read it, with nothing
    of it in the other queries' results: those are the same bits as without it."""
    nh, cfg = 2, _cfg(2, dh)
    lens = [n] * b
    plain, table, q = _attend_case(nh, nh, dh, lens, beams, n - 40, seed=b)
    own = table[1, (n - 1) // 64]
    assert (table == own).sum() == 1                        # the last page of row 1 is its own
    seqs = B.Ragged(dev(table), None, dev(np.array(lens, np.int32)))
    run = lambda p, x: host(B.fg_decode_attention_beams_paged(cfg, nh, beams, dev(x), x.shape[1], b, p, seqs)).reshape(b, nh, dh)
    pages = _upload(plain, cfg)
    good = run(pages, q)
    assert np.isfinite(good).all()
    for value in (np.inf, -np.inf, np.nan):
        odd = q.copy()
        odd[2, dh + dh // 2 + 1] = value                    # row 2, head 1
        got = run(pages, odd)
        assert np.isnan(got[2, 1]).all()
        got[2, 1] = good[2, 1]
        assert np.array_equal(got, good)
    for scales in (pages.k_meta, pages.v_meta):
        for value in (np.inf, np.nan):
            was = float(scales[own, 0])
            scales[own, 0] = value
            got = run(pages, q)
            scales[own, 0] = was
            assert not np.isfinite(got[1, 0]).any()
            got[1, 0] = good[1, 0]
            assert np.array_equal(got, good)


def test_calls_on_another_stream():
    nh, dh, cfg = 3, 64, _cfg(3, 64)
    plain = P.I8Pages(4, nh, dh)
    table = np.array([[1, 3]], np.int32)
    kv = _rows((100, 2 * nh * dh), 1)
    plain.append(table, 0, 0, kv[:, :nh * dh], kv[:, nh * dh:])
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        pages, d = B.KVPages(cfg, 4, int8=True), dev(kv)
        B.fg_kv_append_paged(cfg, d, d[:, nh * dh:], 2 * nh * dh, 1, 100, pages, B.Ragged(dev(table)))
        q = dev(_rows((1, nh * dh), 2))
        got = B.fg_decode_attention_paged(cfg, q, nh * dh, 1, pages, B.Ragged(dev(table), None, dev(np.array([100], np.int32))))
    st.synchronize()
    _same(pages, plain)
    _check_attention(plain, table, host(q), [100], nh, nh, dh, host(got))
