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


def _pool(nh=4, dh=64, n=8, **kw):
    return B.KVPages(B.Cfg(nh * dh, nh, 64, 64, 64), n, device="cpu", **({"int8": True} | kw))


def _seqs(b, ids=None):
    """What the calls read of a Ragged (which wants device tensors)."""
    s = B.Ragged.__new__(B.Ragged)
    s.page_table, s.pos, s.device = torch.zeros((b, 2), dtype=torch.int32), torch.zeros(b, dtype=torch.int32), -1
    s.seq_ids, s.rows = None if ids is None else torch.zeros(ids, dtype=torch.int32), min(b, ids or b)
    s.c = B.fg_ragged(None, None, None, 2, b)
    return s


CFG = B.Cfg(256, 4, 64, 64, 64)
HALF = dict(dtype=torch.float16)


def _calls(pool):
    """Every call that takes a pool of 8-bit pages, with all else in order."""
    q, seqs, ints = torch.zeros((2, 768), **HALF), _seqs(2), lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x = torch.zeros((2, 256), **HALF)
    return {
        "append": lambda: B.fg_kv_append_paged(CFG, q[:, 256:], q[:, 512:], 768, 2, 1, pool, seqs),
        "attention": lambda: B.fg_decode_attention_paged(CFG, q, 768, 2, pool, seqs),
        "beams": lambda: B.fg_decode_attention_beams_paged(CFG, 4, 2, q, 768, 2, pool, seqs),
        "gather": lambda: B.fg_kv_gather_paged(CFG, pool, seqs, 2, 3),
        "reorder": lambda: B.fg_beam_reorder_paged(CFG, [pool], ints(2, 2), ints(2), ints(2), 2, 4),
        "decode": lambda: B.fg_decode_layer_paged(CFG, None, x, pool, seqs),
        "prefill": lambda: B.fg_prefill_layer_paged(CFG, None, x.view(2, 1, 256), pool, seqs),
    }


@pytest.mark.parametrize("call", sorted(_calls(None)))
@pytest.mark.parametrize("kw", [dict(dh=128), dict(nh=2), dict(nh=2, dh=128)])
def test_pools_of_other_heads_are_refused(call, kw):
    """The kernels address a pool by the call's heads and head size: with more than it has, beyond its end."""
    with pytest.raises(AssertionError, match="pages of .* heads of"):
        _calls(_pool(**kw))[call]()


def test_attention_refuses_less_than_its_rows():
    pool, att = _pool(), B.fg_decode_attention_beams_paged
    q = torch.zeros((4, 768), **HALF)
    for seqs in (_seqs(3), _seqs(4, ids=3)):
        with pytest.raises(AssertionError, match="name all 4 rows"):
            att(CFG, 4, 2, q, 768, 4, pool, seqs)
    for bad, stride in ((q[:3].clone(), 768), (q[:, :256], 1024), (q.flatten()[:-520].clone(), 768), (q[:, :248].contiguous(), 256),
                        (q[:, 520:], 768)):
        with pytest.raises(AssertionError, match="q is smaller"):
            att(CFG, 4, 2, bad, stride, 4, pool, _seqs(4))
    with pytest.raises(AssertionError, match="q has to be FP16"):
        att(CFG, 4, 2, q.float(), 768, 4, pool, _seqs(4))
    for out in (torch.zeros((3, 256), **HALF), torch.zeros((4, 255), **HALF)):
        with pytest.raises(AssertionError, match="out is smaller"):
            att(CFG, 4, 2, q, 768, 4, pool, _seqs(4), out=out)
    with pytest.raises(AssertionError, match="out has to be FP16"):
        att(CFG, 4, 2, q, 768, 4, pool, _seqs(4), out=torch.zeros((4, 256)))


def test_rows_that_nobody_names_are_refused():
    pool, q = _pool(), torch.zeros((4, 768), **HALF)
    for seqs in (_seqs(3), _seqs(4, ids=3)):
        for call in (lambda: B.fg_kv_append_paged(CFG, q[:, 256:], q[:, 512:], 768, 4, 1, pool, seqs),
                     lambda: B.fg_decode_attention_paged(CFG, q, 768, 4, pool, seqs)):
            with pytest.raises(AssertionError, match="name all 4 rows"):
                call()


def test_gather_refuses_tensors_that_do_not_hold_its_rows():
    pool, ga = _pool(), B.fg_kv_gather_paged
    k = torch.zeros((2, 3, 256), **HALF)
    with pytest.raises(AssertionError, match="name all 2 rows"):
        ga(CFG, pool, _seqs(1), 2, 3)
    for kw in (dict(k_out=k), dict(v_out=k)):
        with pytest.raises(AssertionError, match="both or none"):
            ga(CFG, pool, _seqs(2), 2, 3, **kw)
    with pytest.raises(AssertionError, match="belongs to the caller's"):
        ga(CFG, pool, _seqs(2), 2, 3, row_stride=256)
    for small, stride in ((k[:, :2].contiguous(), None), (k[:, :, :128].contiguous(), 256), (k, 264)):
        with pytest.raises(AssertionError, match="k_out is smaller"):
            ga(CFG, pool, _seqs(2), 2, 3, small, k, stride)
        with pytest.raises(AssertionError, match="v_out is smaller|k_out is smaller"):
            ga(CFG, pool, _seqs(2), 2, 3, k, small, stride)
    with pytest.raises(AssertionError, match="v_out has to be FP16"):
        ga(CFG, pool, _seqs(2), 2, 3, k, k.float())


def test_pools_over_tensors_of_other_shapes_are_refused():
    """KVPages.of: what the shapes say is what the kernels will address."""
    p8, p16, p4 = _pool(), _pool(int8=False, quantized=False), _pool(int8=False)
    of = lambda p, dtype, **kw: B.KVPages.of(*[kw.get(k, getattr(p, k)) for k in ("k_codes", "k_meta", "v_codes", "v_meta")], dtype)  # noqa: E731
    for p, dtype in ((p8, B.FG_I8P64), (p16, B.FG_F16), (p4, B.FG_Q4G64)):
        with pytest.raises(AssertionError) as e:      # all in order: host tensors are what is refused
            of(p, dtype)
        assert "of the codes" not in str(e.value) and "metas" not in str(e.value)
        for kw in (dict(k_codes=p.k_codes[:, :, :63]), dict(v_codes=p.v_codes[:, :, :3]), dict(v_codes=p.v_codes[..., :5]),
                   dict(v_codes=p.v_codes[:7])):
            with pytest.raises(AssertionError, match="shape of the codes"):
                of(p, dtype, **kw)
        with pytest.raises(AssertionError, match="type of the codes"):
            of(p, dtype, k_codes=p.k_codes.float())
    for p, dtype in ((p8, B.FG_I8P64), (p4, B.FG_Q4G64)):
        with pytest.raises(AssertionError, match="shape of the metas"):
            of(p, dtype, k_meta=p.k_meta[:, :3])
        with pytest.raises(AssertionError, match="type of the metas"):
            of(p, dtype, v_meta=p.v_meta.half())
        with pytest.raises(AssertionError, match="have metas"):
            of(p, dtype, v_meta=None)
    with pytest.raises(AssertionError, match="not a format"):
        of(p4, B.FG_Q4G64_TILED)
