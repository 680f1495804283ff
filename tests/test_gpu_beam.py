"""Beam search on the GPU: selection against binary64, reordering against the host's plain form, and both with the paged
layers as a search runs them."""
import numpy as np
import pytest
import torch

from paper_2303_06865_amd import binding as B
from paper_2303_06865_amd import synth
from tests import plain_i8 as P
from tests.util import assert_close, dev, host

pytestmark = pytest.mark.gpu


def _logits(rows, vocab, seed, std=2.0):
    return (np.random.default_rng(seed).standard_normal((rows, vocab)) * std).astype(np.float32)


def _check_select(x, scores, beams, n_best, done=None, eos=-1, logits=None):
    cfg = B.Cfg(64, 1, 64, x.shape[1], 64)
    d = dev(x) if logits is None else logits
    got = B.fg_beam_select(cfg, d, dev(scores), beams, n_best, done=None if done is None else dev(done), eos=eos)
    gj, gw, gv, gd = (host(t) for t in got)
    want = P.select(x, scores, beams, n_best, done, eos)
    wj, ww, wv, wd = (np.array([[c[k] for c in row] for row in want]) for k in range(4))
    # The values are compared in binary64 on both sides; a row's logarithm of sums is off by less than 2^-20 (its terms are
    # binary32 exponentials) and everything is rounded once, to binary32, at the end
    assert np.array_equal(wv == -np.inf, gv == -np.inf)
    fin = wv > -np.inf
    assert (np.abs(gv[fin] - wv[fin]) <= np.abs(wv[fin]) * 2.0 ** -24 + 2.0 ** -20).all()
    assert np.array_equal(gj, wj) and np.array_equal(gw, ww)
    assert np.array_equal(gd, wd)


@pytest.mark.parametrize("vocab", [1, 7, 64, 1000, 4099, 50272])
@pytest.mark.parametrize("n,beams,n_best", [(1, 1, 1), (1, 4, 4), (3, 5, 10), (2, 16, 32), (7, 2, 3)])
def test_select(vocab, n, beams, n_best):
    r = np.random.default_rng(vocab)
    x = _logits(n * beams, vocab, vocab + beams)
    scores = r.uniform(-30, 0, n * beams).astype(np.float32)
    _check_select(x, scores, beams, n_best)
    done = (r.random(n * beams) < 0.4).astype(np.int32)
    scores[r.random(n * beams) < 0.3] = -np.inf
    _check_select(x, scores, beams, n_best, done, eos=vocab // 2)
    _check_select(x, scores, beams, n_best, None, eos=int(x[0].argmax()))


def test_select_in_place():
    x = _logits(12, 5003, 3)
    r = np.random.default_rng(1)
    scores, done = r.uniform(-9, 0, 12).astype(np.float32), (r.random(12) < 0.4).astype(np.int32)
    cfg = B.Cfg(64, 1, 64, 5003, 64)
    want = [host(t) for t in B.fg_beam_select(cfg, dev(x), dev(scores), 4, done=dev(done), eos=9)]
    ds, dd = dev(scores), dev(done)
    got = B.fg_beam_select(cfg, dev(x), ds, 4, done=dd, eos=9, inplace=True)
    for a, b in zip(got, want):
        assert np.array_equal(host(a), b)
    assert np.array_equal(host(ds), want[2].reshape(-1)) and np.array_equal(host(dd), want[3].reshape(-1))


def test_select_ties_and_forbidden_words():
    """Equal logits in a row, equal rows, rows without a word, -inf, NaN and +inf; more wanted than there are."""
    vocab = 3000
    x = np.zeros((8, vocab), np.float32)                    # all equal: the lowest words win
    x[1] = -np.inf                                          # no word at all
    x[2, 5:] = -np.inf                                      # five words
    x[3] = np.nan
    x[3, 100] = 1.0
    x[4, 2999], x[4, 17] = np.inf, np.inf
    x[5] = -3.4e38
    x[6] = np.repeat(np.arange(vocab // 4), 4)[::-1] * 0.01   # rows of four equals, descending order of the words
    x[7] = x[6]
    for beams, best in ((1, 32), (2, 32), (4, 32), (8, 32), (8, 5)):
        _check_select(x, np.zeros(8, np.float32), beams, best)
        _check_select(x, np.linspace(-1, 0, 8).astype(np.float32), beams, best, eos=17)
    _check_select(x, np.full(8, -np.inf, np.float32), 4, 4)
    _check_select(x, np.array([np.nan, 0, -1, 0, 0, np.nan, 0, 0], np.float32), 4, 8)
    _check_select(x, np.zeros(8, np.float32), 4, 32, np.ones(8, np.int32), eos=0)


def test_select_zeros_of_both_signs_are_equal():
    """-0 is 0: the lowest word wins among them, and the lowest beam among scores of -0 and 0."""
    x = np.zeros((4, 3000), np.float32)
    x[:, ::3] = -0.0
    x[:, 1500:] = -4.0
    for beams, best in ((1, 32), (2, 7), (4, 32)):
        _check_select(x, np.zeros(4, np.float32), beams, best)
    _check_select(x, np.array([-0.0, 0.0, -0.0, 0.0], np.float32), 4, 4, np.ones(4, np.int32), eos=5)


def test_select_where_the_best_lie_together():
    """The best words next to each other, at the ends, and a whole row in ascending or descending order."""
    vocab = 50272
    x = _logits(4, vocab, 1)
    x[0, 20000:20040] += 50 + np.arange(40)
    x[1, :32] += 60
    x[2, -32:] += 60
    x[3] = np.arange(vocab) * 1e-3
    _check_select(x, np.zeros(4, np.float32), 1, 32)
    _check_select(x, np.zeros(4, np.float32), 4, 32)
    x[3] = x[3, ::-1]
    _check_select(x, np.zeros(4, np.float32), 2, 16)


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
def test_select_rows_apart_and_unaligned(shift):
    vocab, rows = 1003, 6
    x = _logits(rows, vocab, shift)
    wide = torch.full((rows * 1010 + 8,), 1e30, device="cuda")
    view = wide[shift:shift + rows * 1010].view(rows, 1010)[:, :vocab]
    view.copy_(dev(x))
    _check_select(x, np.zeros(rows, np.float32), 3, 6, logits=view)


def test_select_rows_far_apart():
    """Rows whose distance in elements passes 2^31 when multiplied out."""
    vocab, ld = 1024, (1 << 30) + 64
    big = torch.empty(2 * ld + vocab, device="cuda")
    view = big.as_strided((3, vocab), (ld, 1))
    x = _logits(3, vocab, 4)
    view.copy_(dev(x))
    _check_select(x, np.zeros(3, np.float32), 3, 6, logits=view)


def test_select_sharp_and_flat_rows():
    """One word has nearly all the weight; all have the same; values far from zero."""
    vocab = 20000
    x = _logits(3, vocab, 5, std=0.01)
    x[0, 777] = 80
    x[1] += 1e4
    x[2] -= 1e4
    _check_select(x, np.zeros(3, np.float32), 3, 8)
    _check_select(x, np.zeros(3, np.float32), 1, 32)


# ---------------------------------------------------------------------------------------------- reordering
def _tree(groups, beams, stride, pos, per_group, seed, shared):
    """Tables whose rows share their first `shared` pages within a group and have pages of their own behind."""
    r = np.random.default_rng(seed)
    table = np.full((groups * beams, stride), -1, np.int32)
    for g in range(groups):
        ids = list(g * per_group + r.permutation(per_group))
        prefix = [ids.pop() for _ in range(shared)]
        for j in range(beams):
            used = -(-int(pos[g * beams + j]) // 64)
            k = min(shared, used)
            table[g * beams + j, :k] = prefix[:k]
            for c in range(k, used):
                table[g * beams + j, c] = ids.pop()
    return table


def _pool(fmt, cfg, n_pages, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = B.KVPages(cfg, n_pages, meta_f16=fmt == "q4h", quantized=fmt != "f16", int8=fmt == "i8")
    for t in (pages.k_codes, pages.v_codes, pages.k_meta, pages.v_meta):
        if t is not None:
            if t.is_floating_point():
                t.normal_(generator=g)
            else:
                t.random_(-128 if fmt == "i8" else 0, 128 if fmt == "i8" else 256, generator=g)
    return pages


def _arrays(pages, fmt):
    """All arrays of a pool with the 64 positions as one axis (2), or [n_pages, nh] scales."""
    out = []
    for t, v in ((pages.k_codes, False), (pages.v_codes, True), (pages.k_meta, False), (pages.v_meta, False)):
        if t is not None:
            a = host(t)
            out.append(a.transpose(0, 1, 2, 4, 3).reshape(a.shape[0], a.shape[1], 64, -1) if v and fmt == "i8" else a)
    return out


@pytest.mark.parametrize("fmt", ["i8", "f16", "q4", "q4h"])
@pytest.mark.parametrize("groups,beams,at,layers", [(1, 4, 130, 1), (3, 2, 64, 2), (2, 8, 100, 3), (2, 16, 127, 1), (5, 3, 1, 2), (1, 5, 0, 1),
                                                   (2, 1, 77, 1)])
@pytest.mark.parametrize("inplace", [False, True])
def test_reorder(fmt, groups, beams, at, layers, inplace):
    nh, dh = 3, 64 if fmt == "q4" else 128
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 4096)
    r = np.random.default_rng(at + beams)
    rows, stride = groups * beams, at // 64 + 2
    shared = at // 128
    per = shared + beams * (at // 64 + 1 - shared) + beams + 1
    pos = np.full(rows, at, np.int32)
    if beams == 8:
        pos[::3] = max(0, at - 70)                       # beams of several lengths
    table = _tree(groups, beams, stride, pos, per, at, shared)
    parents = r.integers(0, beams, rows).astype(np.int32)
    parents[0] = -1                                      # itself
    pools = [_pool(fmt, cfg, groups * per + 3, j) for j in range(layers)]
    before = [_arrays(p, fmt) for p in pools]
    dt, dp = dev(table), dev(pos)
    kw = dict(table_out=dt, pos_out=dp) if inplace else {}
    got_t, got_p, miss = B.fg_beam_reorder_paged(cfg, pools, dt, dp, dev(parents), beams, per, **kw)
    wt, wp, wm, copies = P.reorder(table, pos, parents, beams, per)
    assert np.array_equal(host(got_t), wt) and np.array_equal(host(got_p), wp) and np.array_equal(host(miss), wm)
    for pool, old in zip(pools, before):
        for a, want in zip(_arrays(pool, fmt), old):
            for _, src, dst, n in copies:
                if a.ndim == 2:
                    want[dst] = want[src]
                else:
                    want[dst, :, :n] = want[src, :, :n]
            assert np.array_equal(a.view(np.uint8), want.view(np.uint8))


def test_reorder_shared_begun_page_and_pages_of_others():
    """Right after the prompt: all beams hold the same begun page; in the second group it lies outside the group's own pages."""
    nh, dh = 2, 64
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 4096)
    beams, per = 4, 8
    table = np.array([[3, 5, -1]] * 4 + [[17, 18, -1]] * 4, np.int32)
    pos = np.full(8, 90, np.int32)
    pool = _pool("i8", cfg, 20, 1)
    before = _arrays(pool, "i8")
    parents = np.array([0, 0, 0, 0, 3, 2, 1, 0], np.int32)
    got_t, _, miss = B.fg_beam_reorder_paged(cfg, [pool], dev(table), dev(pos), dev(parents), beams, per)
    wt, _, _, copies = P.reorder(table, pos, parents, beams, per)
    assert np.array_equal(host(got_t), wt) and not host(miss).any() and len(copies) == 7
    assert wt[:4, 1].tolist() == [5, 0, 1, 2] and wt[4:, 1].tolist() == [8, 9, 10, 11]
    for a, want in zip(_arrays(pool, "i8"), before):
        for _, src, dst, n in copies:
            if a.ndim == 2:
                want[dst] = want[src]
            else:
                want[dst, :, :n] = want[src, :, :n]
        assert np.array_equal(a.view(np.uint8), want.view(np.uint8))


def test_reorder_without_room():
    """No free page, a full table, lengths out of range, entries that are no pages: counted, and nothing else is touched."""
    nh, dh = 2, 64
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 4096)
    pool = _pool("f16", cfg, 9, 1)
    before = _arrays(pool, "f16")
    table = np.array([[0, 1], [0, 2], [3, 4], [3, 5], [6, 7], [6, 99]], np.int32)
    pos = np.array([70, 70, 128, 128, 70, 1 << 30], np.int32)
    parents = np.array([0, 0, 1, 0, 1, 0], np.int32)
    for per in (3, 2):
        got_t, got_p, miss = B.fg_beam_reorder_paged(cfg, [pool], dev(table), dev(pos), dev(parents), 2, per)
        wt, wp, wm, copies = P.reorder(table, pos, parents, 2, per)
        assert np.array_equal(host(got_t), wt) and np.array_equal(host(got_p), wp) and np.array_equal(host(miss), wm)
        assert wm.any()
        for a, want in zip(_arrays(pool, "f16"), before):
            for _, src, dst, n in copies:
                want[dst, :, :n] = want[src, :, :n]
            assert np.array_equal(a.view(np.uint8), want.view(np.uint8))


def test_reorder_many_layers_and_long_tables():
    """More layers than one launch takes, more columns than a workgroup has threads, more pages than bits in a few words."""
    nh, dh = 1, 64
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 1000, 4096)
    beams, at, layers = 3, 64 * 700 + 30, 67
    per = 400 + 3 * 301 + 3
    pos = np.full(2 * beams, at, np.int32)
    table = _tree(2, beams, 702, pos, per, 1, 400)
    parents = np.array([2, 2, 0, 1, 1, 1], np.int32)
    k = torch.zeros((layers, 2 * per, nh, 64, dh), dtype=torch.float16, device="cuda")
    k[:, :, 0, 0, 0] = torch.arange(2 * per, device="cuda") % 1000 + torch.arange(layers, device="cuda")[:, None]
    v = k + 1
    want_k, want_v = host(k), host(v)
    pools = [B.KVPages.of(k[j], None, v[j], None, B.FG_F16) for j in range(layers)]
    got_t, _, _ = B.fg_beam_reorder_paged(cfg, pools, dev(table), dev(pos), dev(parents), beams, per)
    wt, _, _, copies = P.reorder(table, pos, parents, beams, per)
    assert np.array_equal(host(got_t), wt) and len(copies) == 3
    for _, src, dst, n in copies:
        want_k[:, dst, :, :n] = want_k[:, src, :, :n]
        want_v[:, dst, :, :n] = want_v[:, src, :, :n]
    assert np.array_equal(host(k), want_k) and np.array_equal(host(v), want_v)


# ---------------------------------------------------------------------------------------------- as they are used
SH = synth.Shape(h1=256, nh=4, h2=512, vocab=2000, max_pos=256, l=2)


def _model():
    cfg = B.Cfg(SH.h1, SH.nh, SH.h2, SH.vocab, SH.max_pos)
    layers = [B.LayerWeights.from_numpy(synth.layer_tensors(SH, 0, j, std=0.08, biases=True, random_ln=True), True) for j in range(SH.l)]
    m = {k: dev(a) for k, a in synth.model_tensors(SH, 0, std=0.08).items()}
    return cfg, layers, m


class _Search:
    """A beam search over paged layers, the way a serving program would write it."""

    def __init__(self, int8, prompts, beams, steps, eos=-1):
        self.cfg, self.layers, self.m = _model()
        n, s = prompts.shape
        self.n, self.s, self.beams, self.eos = n, s, beams, eos
        self.stride = (s + steps) // 64 + 2
        self.per = s // 64 + 1 + beams * (steps // 64 + 2)
        self.pools = [B.KVPages(self.cfg, n * self.per, int8=int8, quantized=int8) for _ in self.layers]
        first = np.full((n, self.stride), -1, np.int32)
        for g in range(n):
            first[g, :s // 64 + 1] = g * self.per + np.arange(s // 64 + 1)
        x = B.fg_embed(self.cfg, self.m["embed"], self.m["pos"], dev(prompts), s, 0).view(n, s, SH.h1)
        ragged = B.Ragged(dev(first))
        for w, pool in zip(self.layers, self.pools):
            x = B.fg_prefill_layer_paged(self.cfg, w, x, pool, ragged)
        self.logits = self._head(x[:, -1].contiguous()).repeat_interleave(beams, 0)
        self.table = dev(np.repeat(first, beams, 0))
        self.pos = torch.full((n * beams,), s, dtype=torch.int32, device="cuda")
        self.scores = torch.full((n, beams), -np.inf, device="cuda")
        self.scores[:, 0] = 0
        self.done = torch.zeros((n * beams,), dtype=torch.int32, device="cuda")
        self.text = torch.zeros((n, beams, 0), dtype=torch.int32, device="cuda")

    def _head(self, x):
        return B.fg_lm_head_greedy(self.cfg, x, self.m["lnf_g"], self.m["lnf_b"], self.m["embed"])[1]

    def step(self):
        par, ids, sc, done = B.fg_beam_select(self.cfg, self.logits, self.scores.flatten(), self.beams, done=self.done if self.eos >= 0 else None,
                                              eos=self.eos)
        self.scores, self.done = sc, done.flatten()
        self.text = torch.cat((torch.gather(self.text, 1, par.long()[..., None].expand(-1, -1, self.text.shape[2])), ids[..., None]), 2)
        B.fg_beam_reorder_paged(self.cfg, self.pools, self.table, self.pos, par.contiguous(), self.beams, self.per, table_out=self.table,
                                pos_out=self.pos)
        x = B.fg_embed_ragged(self.cfg, self.m["embed"], self.m["pos"], ids.contiguous(), self.pos)
        ragged = B.Ragged(self.table, None, self.pos)
        for w, pool in zip(self.layers, self.pools):
            x = B.fg_decode_layer_paged(self.cfg, w, x, pool, ragged, beams=self.beams)
        self.pos += 1
        self.logits = self._head(x)


@pytest.mark.parametrize("beams,s,eos", [(4, 50, -1), (3, 64, -1), (1, 20, -1), (4, 61, 7)])
def test_beam_search_equals_scoring_its_own_texts(beams, s, eos):
    """FP16 pages: what the search says its beams are worth is what the model says, when each text is run through it alone."""
    steps = 9
    prompts = synth.prompt_ids(3, s, SH.vocab, 1).astype(np.int32)
    run = _Search(False, prompts, beams, steps, eos)
    for _ in range(steps):
        run.step()
    text, scores = host(run.text), host(run.scores)
    cfg, layers, m = run.cfg, run.layers, run.m
    for g in range(3):
        for j in range(beams):
            ids = np.concatenate((prompts[g], text[g, j]))[None]
            pool = [B.KVPages(cfg, 2, quantized=False) for _ in layers]
            x = B.fg_embed(cfg, m["embed"], m["pos"], dev(ids), ids.shape[1], 0).view(1, -1, SH.h1)
            for w, p in zip(layers, pool):
                x = B.fg_prefill_layer_paged(cfg, w, x, p, B.Ragged(dev(np.array([[0, 1]], np.int32))))
            lg = host(run._head(x[0, s - 1:-1].contiguous())).astype(np.float64)
            lp = lg - np.log(np.exp(lg - lg.max(1, keepdims=True)).sum(1, keepdims=True)) - lg.max(1, keepdims=True)
            want = 0.0
            for t in range(steps):
                want += lp[t, text[g, j, t]]
                if text[g, j, t] == eos:
                    break
            # every step's logits are off by FP16 activations: measured on the layers' own tests, 1e-2 at most each
            assert abs(scores[g, j] - want) <= 2e-2 * steps
        assert (np.diff(scores[g]) <= 0).all()
        assert len({tuple(t) for t in text[g]}) == beams


def test_beam_search_on_8_bit_pages_and_one_beam_is_greedy():
    prompts = synth.prompt_ids(2, 70, SH.vocab, 3).astype(np.int32)
    run = _Search(True, prompts, 4, 6)
    for _ in range(6):
        run.step()
    assert np.isfinite(host(run.scores)).all() and (host(run.text) >= 0).all()
    one = _Search(True, prompts, 1, 6)
    for _ in range(6):
        one.step()
    pools = [B.KVPages(one.cfg, B.fg_diagonal_pages_needed(2, 70, 6, 2), int8=True) for _ in one.layers]
    m = one.m
    ids, _ = B.fg_generate_diagonal(one.cfg, one.layers, m["embed"], m["pos"], m["lnf_g"], m["lnf_b"], dev(prompts), 6, 2, pools)
    assert np.array_equal(host(ids), host(one.text)[:, 0])


@pytest.mark.parametrize("fmt", ["i8", "f16", "q4"])
def test_layer_of_beams_is_the_layer(fmt):
    """Sharing pages changes what is read, not what comes out: 8-bit pages up to the order of sums (within the suite's bar for
    activations), the others bit for bit."""
    cfg, layers, _ = _model()
    beams, b, at = 4, 8, 150
    stride, per = 3, 2 + 4 * 2
    pos = np.full(b, at, np.int32)
    table = _tree(2, beams, stride, pos, per, 3, 2)
    outs = []
    for shared in (1, beams):
        pool = _pool(fmt, cfg, 2 * per, 5)
        if fmt == "i8":
            pool.k_meta.abs_().mul_(0.02)
            pool.v_meta.abs_().mul_(0.02)
        elif fmt == "q4":
            pool.k_meta.mul_(0.1)
            pool.v_meta.mul_(0.1)
        x = dev(_logits(b, SH.h1, 1, 1.0).astype(np.float16))
        outs.append(host(B.fg_decode_layer_paged(cfg, layers[0], x, pool, B.Ragged(dev(table), None, dev(pos)), beams=shared)))
    if fmt == "i8":
        assert_close(outs[1], outs[0], "beams")
    else:
        assert np.array_equal(outs[0], outs[1])
    cfg_c, w = cfg.c, layers[0].c
    seqs = B.Ragged(dev(table), None, dev(pos))
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    call = lambda n, k: B.lib().fg_decode_layer_beams_paged(B.C.byref(cfg_c), B.C.byref(w), x.data_ptr(), n, k, B.C.byref(pool.c),  # noqa: E731
                                                            B.C.byref(seqs.c), x.data_ptr(), ws.data_ptr(), ws.numel(), None)
    assert call(8, 3) == call(8, 0) == call(8, 17) == B.FG_ERR_SHAPE and call(0, 4) == B.FG_OK


def test_captured_step_replays():
    """Selection, reordering, append and attention in one graph, replayed with the program's own work in between."""
    nh, dh, beams, n = 4, 64, 4, 2
    cfg = B.Cfg(nh * dh, nh, 4 * nh * dh, 3000, 4096)
    per, stride = 2 + beams * 4, 5
    pools = [B.KVPages(cfg, n * per, int8=True) for _ in range(2)]
    r = np.random.default_rng(0)
    first = np.full((n * beams, stride), -1, np.int32)
    first[:, :2] = np.repeat(np.arange(n), beams)[:, None] * per + np.arange(2)
    start = dict(table=dev(first), pos=torch.full((n * beams,), 100, dtype=torch.int32, device="cuda"), scores=torch.zeros(n * beams, device="cuda"))
    state = {k: t.clone() for k, t in start.items()}
    logits = dev(_logits(n * beams, 3000, 1))
    qkv = dev(r.standard_normal((n * beams, 3 * nh * dh)).astype(np.float16))
    outs = [torch.zeros((n * beams, nh * dh), dtype=torch.float16, device="cuda") for _ in pools]
    ws = [B.beam_select_workspace(cfg, n, beams, beams), B.beam_reorder_workspace(n, beams),
          B.decode_attention_beams_workspace(cfg, nh, beams, n * beams, stride)]

    def step():
        par, _, sc, _ = B.fg_beam_select(cfg, logits, state["scores"], beams, ws=ws[0])
        state["scores"].copy_(sc.flatten())
        B.fg_beam_reorder_paged(cfg, pools, state["table"], state["pos"], par, beams, per, ws=ws[1], table_out=state["table"],
                                pos_out=state["pos"])
        seqs = B.Ragged(state["table"], None, state["pos"])
        for pool, out in zip(pools, outs):
            B.fg_kv_append_paged(cfg, qkv[:, nh * dh:], qkv[:, 2 * nh * dh:], 3 * nh * dh, n * beams, 1, pool, seqs)
            B.fg_decode_attention_beams_paged(cfg, nh, beams, qkv, 3 * nh * dh, n * beams, pool, seqs, rows_bias=1, ws=ws[2], out=out)
        state["pos"] += 1

    def reset():
        for k, t in start.items():
            state[k].copy_(t)
        for p in pools:
            for t in (p.k_codes, p.v_codes, p.k_meta, p.v_meta):
                t.zero_()
        for p in pools:
            B.fg_kv_append_paged(cfg, rows, rows, nh * dh, n, 100, p, B.Ragged(heads))

    rows = dev(r.standard_normal((n * 100, nh * dh)).astype(np.float16))
    heads = dev(first[::beams])
    seen = []
    reset()
    for k in range(4):
        logits.copy_(dev(_logits(n * beams, 3000, k)))
        step()
        torch.cuda.synchronize()
        seen.append([host(t).copy() for t in (state["table"], state["pos"], state["scores"], *outs)])
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    reset()
    for k in range(4):
        logits.copy_(dev(_logits(n * beams, 3000, k)))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((state["table"], state["pos"], state["scores"], *outs), seen[k]):
            assert np.array_equal(host(got), want), k
