"""The operators of beam search over a paged cache held in 8 bits, and how their speed and results are looked at.

A case is a dict of plain values; its "kind" names the operator:

  append   rows of keys and values into 8-bit pages (one scale per page, head and tensor), then the last rows read back
  gather   rows of a paged cache read back as FP16
  attend   one token's attention over 8-bit pages; rows come in groups of `beams` that share the pages of their prefix
  select   the best continuations over the beams of a sequence and the vocabulary
  reorder  the page tables behind the beams chosen, with copies of the pages that two beams would write to

Heads and head sizes are those of the OPT models that bench.py runs, or generic where cache heads are shared by query heads.
Where `own` is false the plain form runs: elementary torch operations in 32 bits (64 for the scores of the selection, which are
compared with each other).
"""
import math

import numpy as np
import torch

own = False

PAGE = 64        # positions a page holds
VOCAB = 50272    # of the OPT models
FLT_MAX = 3.4028234663852886e38

HEADS = {"125m": (12, 12, 64), "6.7b": (32, 32, 128), "30b": (56, 56, 128), "175b": (96, 96, 128),
         "grouped": (32, 8, 128)}   # query heads, cache heads, head size


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decode step of 64 sequences of mixed lengths: one new row each, into pages that are mostly begun
        dict(name="append_token_6.7b_b64", kind="append", heads="6.7b", b=64, s=1, t=1900, back=16),
        # prompts of 500 tokens stored at once
        dict(name="append_prompt_6.7b_16x500", kind="append", heads="6.7b", b=16, s=500, t=0, back=500),
        # eight conversations moved out of the pool
        dict(name="gather_6.7b_i8_8x1500", kind="gather", heads="6.7b", fmt="i8", b=8, s=1500),
        # the same from the 4.5-bit pages of a larger model
        dict(name="gather_30b_q4h_16x400", kind="gather", heads="30b", fmt="q4h", b=16, s=400),
        # one short sequence of a small model: launches and latency
        dict(name="attend_125m_b1_t200", kind="attend", heads="125m", groups=1, beams=1, t=200, tail=0, mixed=False),
        # one very long sequence, four query heads on each cache head
        dict(name="attend_grouped_b1_t32768", kind="attend", heads="grouped", groups=1, beams=1, t=32768, tail=0, mixed=False),
        # continuous batching: 64 sequences of mixed lengths
        dict(name="attend_6.7b_b64_t2047", kind="attend", heads="6.7b", groups=64, beams=1, t=2047, tail=0, mixed=True),
        # beam search on the largest model: 16 prompts of 512 tokens, four beams each, 30 generated tokens
        dict(name="attend_beams_175b_16x4", kind="attend", heads="175b", groups=16, beams=4, t=542, tail=30, mixed=False),
        # one sequence, four beams
        dict(name="select_1x4", kind="select", groups=1, beams=4, n_best=4, vocab=VOCAB, done=False, masked=0.0, first=False),
        # 64 sequences, eight beams, twice as many candidates as beams, so that finished ones can be set aside
        dict(name="select_64x8_best16", kind="select", groups=64, beams=8, n_best=16, vocab=VOCAB, done=True, masked=0.01, first=False),
        # the smallest model, one sequence
        dict(name="reorder_125m_1x4_l12", kind="reorder", heads="125m", fmt="i8", groups=1, beams=4, t=600, tail=40, layers=12),
        # many sequences; eight layers' pools
        dict(name="reorder_6.7b_24x4_l8", kind="reorder", heads="6.7b", fmt="i8", groups=24, beams=4, t=548, tail=36, layers=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "gather", "attend", "attend", "select", "reorder"])
    if kind == "append":
        heads = rng.choice(["125m", "6.7b", "30b", "grouped"])
        elems = HEADS[heads][1] * HEADS[heads][2]
        if rng.random() < 0.5:
            b, s, t = _log(rng, 1, 96), 1, _log(rng, 1, 2000)
        else:   # prompts, or what continues them
            s = _log(rng, 2, 700)
            b, t = max(1, min(_log(rng, 1, 32), 32000000 // (s * elems))), rng.choice([0, _log(rng, 1, 500)])
        return dict(kind=kind, heads=heads, b=b, s=s, t=t, back=s if s > 1 else 16)
    if kind == "gather":
        heads = rng.choice(["125m", "6.7b", "30b"])
        elems = HEADS[heads][1] * HEADS[heads][2]
        s = _log(rng, 1, 2000)
        return dict(kind=kind, heads=heads, fmt=rng.choice(["i8", "i8", "q4", "q4h", "f16"]), s=s,
                    b=max(1, min(_log(rng, 1, 64), 48000000 // (s * elems))))
    if kind == "attend":
        heads = rng.choice(["125m", "6.7b", "30b", "grouped"])
        elems = HEADS[heads][1] * HEADS[heads][2]
        beams = rng.choice([1, 1, 2, 3, 4, 6])
        t = _log(rng, 1, 4000)
        groups = max(1, min(_log(rng, 1, 64), 250000000 // (beams * t * elems)))
        return dict(kind=kind, heads=heads, groups=groups, beams=beams, t=t, tail=min(t, rng.randint(0, 90)) if beams > 1 else 0,
                    mixed=rng.random() < 0.5)
    if kind == "select":
        vocab = rng.choice([VOCAB, _log(rng, 500, 60000)])
        beams = rng.randint(1, 8)
        return dict(kind=kind, groups=_log(rng, 1, 60), beams=beams, n_best=rng.choice([beams, 2 * beams]), vocab=vocab,
                    done=rng.random() < 0.4, masked=rng.choice([0.0, 0.3]), first=rng.random() < 0.2)
    heads = rng.choice(["125m", "6.7b"])
    t = _log(rng, 65, 1200)
    return dict(kind=kind, heads=heads, fmt=rng.choice(["i8", "f16"]), groups=_log(rng, 1, 12), beams=rng.randint(2, 8), t=t,
                tail=min(t, rng.randint(1, 70)), layers=rng.randint(1, 4))


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _pool(fmt, n_pages, nh, dh, g, layers=None):
    """Pages as rows of about unit spread leave them.  8-bit: key codes [.., nh, 64, dh]; value codes [.., nh, 4, dh, 16], 16
    positions of one head dimension next to each other; scales [.., nh]."""
    lead = (n_pages, nh) if layers is None else (layers, n_pages, nh)
    half = torch.float16

    def codes(shape):
        x = torch.empty(shape, dtype=torch.int8, device="cuda")
        flat = x.view(-1)
        for a in range(0, flat.numel(), 1 << 28):
            z = min(flat.numel(), a + (1 << 28)) - a
            flat[a:a + z] = (torch.randn(z, dtype=half, device="cuda", generator=g) * 32).clamp_(-127, 127).round_().to(torch.int8)
        return x

    if fmt == "i8":
        scale = lambda: torch.empty(lead, device="cuda").uniform_(0.027, 0.036, generator=g)  # noqa: E731
        return dict(kc=codes(lead + (PAGE, dh)), km=scale(), vc=codes(lead + (4, dh, 16)), vm=scale())
    if fmt == "f16":
        rows = lambda: torch.randn(lead + (PAGE, dh), dtype=half, device="cuda", generator=g)  # noqa: E731
        return dict(kc=rows(), km=None, vc=rows(), vm=None)
    mt = half if fmt == "q4h" else torch.float32
    pack = lambda: torch.randint(0, 256, lead + (PAGE, dh // 2), dtype=torch.uint8, device="cuda", generator=g)  # noqa: E731

    def pairs():
        m = torch.empty(lead + (PAGE, dh // 64, 2), device="cuda")
        m[..., 0].uniform_(-3.0, -1.5, generator=g)
        m[..., 1].uniform_(0.25, 0.4, generator=g)
        return m.to(mt)

    return dict(kc=pack(), km=pairs(), vc=pack(), vm=pairs())


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _lengths(case, r, n):
    t = case["t"]
    if case.get("mixed"):
        x = r.integers(1, t + 1, n)
        x[r.integers(n)] = t
        return x
    return np.full(n, t)


def prepare(case, seed):
    r = np.random.default_rng([int(seed), 101])
    g = _gen(seed)
    kind = case["kind"]
    st = dict(case=dict(case))
    if kind == "select":
        rows, vocab = case["groups"] * case["beams"], case["vocab"]
        x = torch.randn((rows, vocab), device="cuda", generator=g).mul_(1.7)
        peaks = torch.randint(0, vocab, (rows, 24), device="cuda", generator=g)
        x.scatter_add_(1, peaks, torch.empty((rows, 24), device="cuda").uniform_(4.0, 11.0, generator=g))   # what a trained model's rows look like
        if case["masked"]:
            x.masked_fill_(torch.rand(x.shape, device="cuda", generator=g) < case["masked"], -math.inf)
            if rows > 2:
                x[int(r.integers(rows))] = -math.inf   # a beam whose words are all forbidden
        sc = torch.empty(rows, device="cuda").uniform_(-40.0, -5.0, generator=g)
        if case["first"]:   # the first step: the beams are still the same, only one of them counts
            sc.view(-1, case["beams"])[:, 1:] = -math.inf
        done = torch.rand(rows, device="cuda", generator=g) < 0.2 if case["done"] else None
        st.update(logits=x, scores=sc, done=None if done is None else done.to(torch.int32), eos=2)
        return st

    nh, nkv, dh = HEADS[case["heads"]]
    st.update(nh=nh, nkv=nkv, dh=dh, scale=1.0 / math.sqrt(dh))
    if kind == "append":
        b, s = case["b"], case["s"]
        low = case["back"] - s   # what is read back ends with the last new row
        pos = r.integers(low, max(low, case["t"]) + 1, b) if s == 1 else np.full(b, case["t"])
        stride = (max(low, case["t"]) + s + PAGE - 1) // PAGE + 1
        st.update(pool=_pool("i8", b * stride, nkv, dh, g), table=_int(r.permutation(b * stride).reshape(b, stride)), pos=_int(pos))
        st["qkv"] = torch.randn((b * s, (nh + 2 * nkv) * dh), dtype=torch.float16, device="cuda", generator=g)
        st["back"] = case["back"]
        st["back_pos"] = _int(pos + s - case["back"])
        return st
    if kind == "gather":
        b, s = case["b"], case["s"]
        pos = r.integers(0, 200, b)
        stride = (200 + s + PAGE - 1) // PAGE
        st.update(pool=_pool(case["fmt"], b * stride, nkv, dh, g), table=_int(r.permutation(b * stride).reshape(b, stride)), pos=_int(pos))
        return st
    groups, beams, tail = case["groups"], case["beams"], case["tail"]
    if kind == "attend":
        n = _lengths(case, r, groups)
        stride = int((n.max() + PAGE - 1) // PAGE)
        ids = r.permutation(groups * beams * stride)   # pages of the beams' own tails; the prefix of a group is its first beam's
        table = ids.reshape(groups, beams, stride).copy()
        for q in range(groups):
            table[q, :, :max(0, int(n[q]) - tail) // PAGE] = table[q, 0, :max(0, int(n[q]) - tail) // PAGE]
        st.update(pool=_pool("i8", groups * beams * stride, nkv, dh, g), table=_int(table.reshape(groups * beams, stride)),
                  pos=_int(np.repeat(n, beams)))
        st["q"] = torch.randn((groups * beams, (nh + 2 * nkv) * dh), dtype=torch.float16, device="cuda", generator=g) * 2
        return st
    # reorder: every group has its own range of pages
    layers, t = case["layers"], case["t"]
    stride = t // PAGE + 2
    shared = (t - tail) // PAGE
    per_group = shared + beams * (stride - shared) + beams
    table = np.full((groups, beams, stride), -1)
    for q in range(groups):
        ids = q * per_group + r.permutation(per_group)
        used = (t + PAGE - 1) // PAGE
        table[q, :, :shared] = ids[:shared]
        table[q, :, shared:used] = ids[shared:shared + beams * (used - shared)].reshape(beams, used - shared)
    st.update(pool=_pool(case["fmt"], groups * per_group, nkv, dh, g, layers=layers), per_group=per_group,
              table=_int(table.reshape(groups * beams, stride)), pos=_int(np.full(groups * beams, t)),
              parents=_int(r.integers(0, beams, groups * beams)))
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _rows_of(st, codes, meta, page, off, values):
    """Rows `off` of pages `page` (index tensors of one shape) as [.., heads, dh] in 32 bits."""
    fmt = st["case"].get("fmt", "i8")
    if fmt == "f16":
        return codes[page, :, off].float()
    if fmt == "i8":
        c = codes[page, :, off >> 4, :, off & 15] if values else codes[page, :, off]
        return c.float() * meta[page].unsqueeze(-1)
    c = codes[page, :, off]
    c = torch.stack((c & 15, c >> 4), -1).flatten(-2).float()
    m = meta[page, :, off].float()
    return (c.unflatten(-1, (-1, 64)) * m[..., 1:2] + m[..., 0:1]).flatten(-2)


def _gathered(st, pos, s):
    at = pos.long()[:, None] + torch.arange(s, device="cuda")
    page, off = torch.gather(st["table"].long(), 1, at >> 6), at & 63
    p = st["pool"]
    return [_rows_of(st, p[c], p[m], page, off, c == "vc").half().flatten(-2) for c, m in (("kc", "km"), ("vc", "vm"))]


def _append_one(st, codes, scales, x, values):
    """x [b, s, heads, dh] into the pages of its rows: the scale of a page grows with its rows and is begun anew at row 0."""
    b, s, nh, dh = x.shape
    pos = st["pos"].long()
    first = pos >> 6
    slots = (s + 126) // PAGE + 1
    at = pos[:, None] + torch.arange(s, device="cuda")
    # rows into a [b, slots, 64] frame of the pages they touch
    frame = torch.zeros((b, slots * PAGE, nh, dh), device="cuda")
    fresh = torch.zeros((b, slots * PAGE), dtype=torch.bool, device="cuda")
    col = at - (first << 6)[:, None]
    row = torch.arange(b, device="cuda")[:, None]
    frame[row, col] = x.float()
    fresh[row, col] = True
    frame, fresh = frame.view(b, slots, PAGE, nh, dh), fresh.view(b, slots, PAGE)
    touched = fresh.any(-1)
    slot = (first[:, None] + torch.arange(slots, device="cuda")).clamp(max=st["table"].shape[1] - 1)
    page = torch.where(touched, torch.gather(st["table"].long(), 1, slot), codes.shape[0])   # one page more takes what is no page
    pad = lambda v: torch.cat((v, torch.zeros_like(v[:1])))  # noqa: E731
    c_all, s_all = pad(codes), pad(scales)
    old_c = c_all[page].float()                            # [b, slots, heads, ...]
    if values:
        old_c = old_c.transpose(-1, -2).flatten(3, 4)      # [.., heads, 64, dh]
    old_s = torch.where(fresh[:, :, :1], 0.0, s_all[page])
    top = frame.abs().amax((2, 4)) / torch.tensor(127.0, device="cuda")
    new_s = torch.maximum(old_s, top)
    ratio = torch.where(new_s > old_s, old_s / new_s, 1.0)
    inv = torch.where(new_s > 0, 1.0 / new_s, 0.0)
    new = torch.where(fresh[:, :, None, :, None], torch.round(frame.transpose(2, 3) * inv[..., None, None]),
                      torch.round(old_c * ratio[..., None, None]))
    if values:
        new = new.unflatten(3, (4, 16)).transpose(-1, -2)
    c_all[page] = new.to(torch.int8)
    s_all[page] = new_s
    codes.copy_(c_all[:-1])
    scales.copy_(s_all[:-1])


def _plain_append(st):
    c, p = st["case"], st["pool"]
    nh, nkv, dh = st["nh"], st["nkv"], st["dh"]
    kv = st["qkv"].view(c["b"], c["s"], nh + 2 * nkv, dh)
    _append_one(st, p["kc"], p["km"], kv[:, :, nh:nh + nkv], False)
    _append_one(st, p["vc"], p["vm"], kv[:, :, nh + nkv:], True)
    return _gathered(st, st["back_pos"], st["back"]) + [p["km"], p["vm"]]


def _plain_attend(st):
    nh, nkv, dh = st["nh"], st["nkv"], st["dh"]
    table, p, n = st["table"].long(), st["pool"], st["pos"].long()
    b, t = table.shape[0], table.shape[1] * PAGE
    k = (p["kc"][table].float() * p["km"][table][..., None, None]).transpose(1, 2).reshape(b, nkv, t, dh)
    v = p["vc"][table].float() * p["vm"][table][..., None, None, None]
    v = v.transpose(-1, -2).flatten(3, 4).transpose(1, 2).reshape(b, nkv, t, dh)
    q = st["q"][:, :nh * dh].float().reshape(b, nkv, nh // nkv, dh)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * st["scale"]
    x = x.masked_fill(torch.arange(t, device="cuda") >= n[:, None, None, None], -math.inf)
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return (torch.matmul(e, v) / e.sum(-1, keepdim=True)).reshape(b, nh * dh).half()


def _plain_select(st):
    c = st["case"]
    beams, vocab, n_best = c["beams"], c["vocab"], c["n_best"]
    x = st["logits"].double()
    x = torch.where(torch.isnan(x), -math.inf, x.clamp(max=FLT_MAX))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    v = st["scores"].double()[:, None] + (x - (torch.log(torch.exp(x - m).sum(-1, keepdim=True)) + m))
    v = torch.where(x == -math.inf, -math.inf, v)
    if st["done"] is not None:
        word = torch.arange(vocab, device="cuda")
        v = torch.where(st["done"][:, None] != 0, torch.where(word == st["eos"], st["scores"].double()[:, None], -math.inf), v)
    v, i = torch.sort(v.view(-1, beams * vocab), dim=-1, descending=True, stable=True)
    v, i = v[:, :n_best], i[:, :n_best]
    if v.shape[1] < n_best:
        short = (v.shape[0], n_best - v.shape[1])
        v, i = torch.cat((v, v.new_full(short, -math.inf)), 1), torch.cat((i, i.new_zeros(short)), 1)
    none = v == -math.inf
    parent, word = torch.where(none, -1, i // vocab), torch.where(none, -1, i % vocab)
    out = {"parents": parent.int(), "ids": word.int(), "scores": v.float()}
    if st["done"] is not None:
        was = torch.gather(st["done"].view(-1, beams), 1, parent.clamp(min=0)) != 0
        out["done"] = (was | (word == st["eos"]) | none).int()
    return out


def _plain_reorder(st):
    c = st["case"]
    beams, per = c["beams"], st["per_group"]
    table, pos = st["table"].long().view(-1, beams, st["table"].shape[1]), st["pos"].long().view(-1, beams)
    groups, _, stride = table.shape
    par = st["parents"].long().view(-1, beams)
    pos = torch.gather(pos, 1, par)
    slot = torch.arange(stride, device="cuda")
    held = slot < ((pos + 63) >> 6)[..., None]
    table = torch.where(held, torch.gather(table, 1, par[..., None].expand(-1, -1, stride)), -1)
    # the page of the next row: the first beam that holds a begun page keeps it, the others take free ones
    at = pos >> 6
    begun = (pos & 63) != 0
    page = torch.gather(table, 2, at[..., None])[..., 0]
    same = (page[:, :, None] == page[:, None, :]) & begun[:, :, None] & begun[:, None, :]
    earlier = torch.ones((beams, beams), dtype=torch.bool, device="cuda").tril(-1)
    takes = ~begun | (same & earlier).any(-1)
    own_first = (torch.arange(groups, device="cuda") * per)[:, None]
    used = torch.zeros((groups, per + 1), dtype=torch.int32, device="cuda")
    local = torch.where(table >= 0, table - own_first[..., None], per).flatten(1)
    used.scatter_(1, local, 1)
    free = torch.sort(used[:, :per], dim=1, stable=True)[1]   # pages that nobody holds come first, the lowest first
    new = torch.gather(free, 1, (takes.long().cumsum(1) - 1).clamp(min=0)) + own_first
    dst = torch.where(takes, new, page)
    table.scatter_(2, at[..., None], dst[..., None])
    # copies in every layer: whole sixteens of rows, as far as the page is filled
    src = torch.where(begun, page, dst).flatten()
    dst = dst.flatten()
    filled = torch.where(begun & takes, ((pos & 63) + 15) & ~15, 0).flatten()
    row = torch.arange(PAGE, device="cuda")
    p = st["pool"]
    outs = []
    for name in ("kc", "vc"):
        t = p[name]
        m = row < filled[:, None]
        m = m.view(1, -1, 1, 4, 1, 16) if name == "vc" and c["fmt"] == "i8" else m.view(1, -1, 1, PAGE, 1)
        t[:, dst] = torch.where(m, t[:, src], t[:, dst])
        outs.append(t)
    for name in ("km", "vm"):
        if p[name] is not None:
            t = p[name]
            t[:, dst] = torch.where((filled > 0).view(1, -1, 1), t[:, src], t[:, dst])
            outs.append(t)
    return [table.view(-1, stride).int(), pos.flatten().int()] + outs


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handles(st):
    """What a program makes once beside its buffers: the model's shape, the pools, the rows' description, scratch."""
    from paper_2303_06865_amd import binding as B
    h = {"B": B}
    c = st["case"]
    if c["kind"] == "select":
        h["cfg"] = B.Cfg(64, 1, 64, c["vocab"], 64)
        h["ws"] = B.beam_select_workspace(h["cfg"], c["groups"], c["beams"], c["n_best"])
        return h
    nh, nkv, dh = st["nh"], st["nkv"], st["dh"]
    h["cfg"] = B.Cfg(nh * dh, nh, 4 * nh * dh, VOCAB, 1 << 20)
    h["kv_cfg"] = B.Cfg(nkv * dh, nkv, 4 * nkv * dh, VOCAB, 1 << 20)
    p, fmt = st["pool"], c.get("fmt", "i8")
    dtype = {"i8": B.FG_I8P64, "f16": B.FG_F16, "q4": B.FG_Q4G64, "q4h": B.FG_Q4G64_H16}[fmt]
    of = lambda j: B.KVPages.of(*(None if p[k] is None else (p[k] if j is None else p[k][j]) for k in ("kc", "km", "vc", "vm")), dtype)  # noqa: E731
    if c["kind"] == "reorder":
        h["pages"] = [of(j) for j in range(c["layers"])]
        h["ws"] = B.beam_reorder_workspace(c["groups"], c["beams"])
        return h
    h["pages"], h["seqs"] = of(None), B.Ragged(st["table"], None, st["pos"])
    if c["kind"] == "append":
        h["back"] = B.Ragged(st["table"], None, st["back_pos"])
    if c["kind"] == "attend":
        h["ws"] = B.decode_attention_beams_workspace(h["cfg"], nkv, c["beams"], st["q"].shape[0], st["table"].shape[1])
    return h


def _own(st):
    if "handles" not in st:
        st["handles"] = _handles(st)
    h, c = st["handles"], st["case"]
    B, kind = h["B"], c["kind"]
    if kind == "append":
        nh, nkv, dh, p = st["nh"], st["nkv"], st["dh"], st["pool"]
        qkv = st["qkv"]
        B.fg_kv_append_paged(h["kv_cfg"], qkv[:, nh * dh:], qkv[:, (nh + nkv) * dh:], qkv.shape[1], c["b"], c["s"], h["pages"], h["seqs"])
        return list(B.fg_kv_gather_paged(h["kv_cfg"], h["pages"], h["back"], c["b"], st["back"])) + [p["km"], p["vm"]]
    if kind == "gather":
        return list(B.fg_kv_gather_paged(h["kv_cfg"], h["pages"], h["seqs"], c["b"], c["s"]))
    if kind == "attend":
        q = st["q"]
        return B.fg_decode_attention_beams_paged(h["cfg"], st["nkv"], c["beams"], q, q.shape[1], q.shape[0], h["pages"], h["seqs"], ws=h["ws"])
    if kind == "select":
        got = B.fg_beam_select(h["cfg"], st["logits"], st["scores"], c["beams"], c["n_best"], done=st["done"], eos=st["eos"], ws=h["ws"])
        return dict(zip(("parents", "ids", "scores", "done"), got if st["done"] is not None else got[:3]))
    p = st["pool"]
    table, pos, _ = B.fg_beam_reorder_paged(h["kv_cfg"], h["pages"], st["table"], st["pos"], st["parents"], c["beams"], st["per_group"], ws=h["ws"])
    return [table, pos] + [p[k] for k in ("kc", "vc", "km", "vm") if p[k] is not None]


def run(st):
    if own:
        return _own(st)
    kind = st["case"]["kind"]
    if kind == "append":
        return _plain_append(st)
    if kind == "gather":
        return _gathered(st, st["pos"], st["case"]["s"])
    if kind == "attend":
        return _plain_attend(st)
    return _plain_select(st) if kind == "select" else _plain_reorder(st)


# ------------------------------------------------------------------------------------------------ work and definition
def work(case):
    kind = case["kind"]
    if kind == "select":
        rows = case["groups"] * case["beams"]
        return {"bytes": rows * case["vocab"] * 4 + rows * 8 + case["groups"] * case["n_best"] * 16, "flops": 4 * rows * case["vocab"]}
    nh, nkv, dh = HEADS[case["heads"]]
    per_row = {"i8": 1.0, "f16": 2.0, "q4": 0.625, "q4h": 0.5625}[case.get("fmt", "i8")] * 2 * nkv * dh   # keys and values of a row
    scales = 2 * nkv * 4 if case.get("fmt", "i8") == "i8" else 0                                            # of a page
    if kind == "append":
        rows, back = case["b"] * case["s"], case["b"] * case["back"]
        pages = case["b"] * -(-case["s"] // PAGE)
        return {"bytes": rows * (4 * nkv * dh + per_row) + back * (per_row + 4 * nkv * dh) + 2 * pages * scales, "flops": 4 * rows * nkv * dh}
    if kind == "gather":
        rows = case["b"] * case["s"]
        return {"bytes": rows * (per_row + 4 * nkv * dh) + -(-rows // PAGE) * scales, "flops": 4 * rows * nkv * dh}
    groups, beams, t, tail = case["groups"], case["beams"], case["t"], case["tail"]
    if kind == "attend":
        t = (t + 1) / 2 if case["mixed"] else t
        shared = max(0, t - tail) // PAGE * PAGE if beams > 1 else 0
        rows = groups * (shared + beams * (t - shared))
        return {"bytes": rows * per_row + rows / PAGE * scales + 4 * groups * beams * nh * dh, "flops": 4 * groups * beams * t * nh * dh}
    # of four beams with parents drawn freely, about this share has a begun page that an earlier one keeps
    copied = groups * sum(1 - (1 - 1 / beams) ** i for i in range(beams)) if case["t"] % PAGE else 0
    return {"bytes": case["layers"] * copied * 2 * (case["t"] % PAGE * per_row + scales) + 8 * groups * beams * (case["t"] // PAGE + 2), "flops": 0}


def _definition(st, name, page, off):
    """Rows of a paged cache in 64 bits: [n, heads, dh] of page[i], off[i]."""
    p, fmt = st["pool"], st["case"].get("fmt", "i8")
    c, m = p[name + "c"], p[name + "m"]
    if fmt == "f16":
        return c[page, :, off].double()
    if fmt == "i8":
        c = c if name == "k" else c.permute(0, 1, 2, 4, 3).reshape(c.shape[0], c.shape[1], PAGE, -1)
        return c[page, :, off].double() * m[page].double()[..., None]
    c, m = c[page, :, off], m[page, :, off].double()
    dh = 2 * c.shape[-1]
    d = torch.arange(dh, device="cuda")
    nib = (c[..., d // 2].long() >> (4 * (d % 2))) & 15
    return m[..., d // 64, 0] + nib.double() * m[..., d // 64, 1]


def exact(case, seed):
    kind = case["kind"]
    if kind == "reorder":
        return None   # numbers of pages, and bytes moved
    st = prepare(case, seed)
    if kind == "select":
        x, beams, n = st["logits"].double(), case["beams"], case["n_best"]
        rows = []
        for j in range(x.shape[0]):
            if st["done"] is not None and int(st["done"][j]):
                rows.append(st["scores"][j:j + 1].double())
                continue
            best = torch.topk(x[j], min(n, x.shape[1]))[0]
            v = st["scores"][j].double() + best - torch.logsumexp(x[j], 0)
            rows.append(torch.where(best == -math.inf, -math.inf, v))
        out = x.new_full((case["groups"], n), -math.inf)
        for q in range(case["groups"]):
            v = torch.cat(rows[q * beams:(q + 1) * beams]).sort(descending=True)[0][:n]
            out[q, :v.numel()] = v
        got = {"parents": None, "ids": None, "scores": out}
        return got if st["done"] is None else {**got, "done": None}
    nh, nkv, dh = HEADS[case["heads"]]
    table = st["table"].long()
    if kind == "gather":
        outs = {"k": [], "v": []}
        for i in range(case["b"]):
            at = int(st["pos"][i]) + torch.arange(case["s"], device="cuda")
            for name in outs:
                outs[name].append(_definition(st, name, table[i, at // PAGE], at % PAGE).flatten(1))
        return [torch.stack(outs["k"]), torch.stack(outs["v"])]
    if kind == "append":
        b, s, back = case["b"], case["s"], case["back"]
        kv = st["qkv"].view(b, s, nh + 2 * nkv, dh).double()
        outs, scales = {"k": [], "v": []}, {"k": st["pool"]["km"].double().clone(), "v": st["pool"]["vm"].double().clone()}
        for name, lo in (("k", nh), ("v", nh + nkv)):
            for i in range(b):
                p0, start = int(st["pos"][i]), int(st["back_pos"][i])
                held = torch.arange(start, start + back, device="cuda")
                res = _definition(st, name, table[i, held // PAGE], held % PAGE)
                x = kv[i, :, lo:lo + nkv]
                for a in range(p0 // PAGE, (p0 + s - 1) // PAGE + 1):
                    j0, j1 = max(p0, a * PAGE), min(p0 + s, (a + 1) * PAGE)
                    part, page = x[j0 - p0:j1 - p0], int(table[i, a])
                    was = scales[name][page] if j0 % PAGE else torch.zeros(nkv, dtype=torch.float64, device="cuda")
                    now = torch.maximum(was, part.abs().amax((0, 2)) / 127)
                    scales[name][page] = now
                    step = torch.where(now > 0, now, 1.0)[:, None]
                    here = (held // PAGE == a)
                    old = res[here]
                    res[here] = torch.where((now > was)[:, None], torch.round(old / step) * step, old)
                    new = torch.round(part / step) * step
                    fit = (held >= j0) & (held < j1)
                    res[fit] = new[held[fit] - j0]
                outs[name].append(res.flatten(1))
        return [torch.stack(outs["k"]), torch.stack(outs["v"]), scales["k"], scales["v"]]
    out = []
    for i in range(table.shape[0]):
        n = int(st["pos"][i])
        at = torch.arange(n, device="cuda")
        k, v = (_definition(st, name, table[i, at // PAGE], at % PAGE) for name in ("k", "v"))
        q = st["q"][i, :nh * dh].double().view(nkv, nh // nkv, dh)
        w = torch.softmax(torch.matmul(q, k.permute(1, 2, 0)) / math.sqrt(dh), -1)
        out.append(torch.matmul(w, v.permute(1, 0, 2)).reshape(nh * dh))
    return torch.stack(out)
