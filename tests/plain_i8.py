"""Plain implementations that the tests of 8-bit pages and beam search compare with: numpy, written from the definitions
in include/fg.h, in binary64 except where the format itself is defined by binary32 steps."""
import numpy as np

PAGE = 64


class I8Pages:
    """The host's copy of a pool: keys [n, nh, 64, dh], values here in the order of positions too [n, nh, 64, dh]."""

    def __init__(self, n_pages, nh, dh, seed=None):
        self.n, self.nh, self.dh = n_pages, nh, dh
        shape = (n_pages, nh, PAGE, dh)
        if seed is None:
            self.codes = [np.zeros(shape, np.int8), np.zeros(shape, np.int8)]
            self.scales = [np.zeros((n_pages, nh), np.float32), np.zeros((n_pages, nh), np.float32)]
        else:
            r = np.random.default_rng(seed)
            self.codes = [np.clip(np.rint(r.standard_normal(shape) * 32), -127, 127).astype(np.int8) for _ in range(2)]
            self.scales = [r.uniform(0.02, 0.05, (n_pages, nh)).astype(np.float32) for _ in range(2)]

    def store(self, page, lo, k, v):
        """Rows k, v [n, nh, dh] FP16 at rows lo .. of a page."""
        for t, x in enumerate((k, v)):
            x = x.astype(np.float32).transpose(1, 0, 2)                       # [nh, n, dh]
            n = x.shape[1]
            top = (np.abs(x).max((1, 2)) / np.float32(127)).astype(np.float32)
            old = self.scales[t][page] if lo else np.zeros(self.nh, np.float32)
            now = np.maximum(old, top)
            c = self.codes[t][page]
            for h in range(self.nh):
                if lo and now[h] > old[h]:
                    c[h] = np.rint(c[h].astype(np.float32) * np.float32(old[h] / now[h])).astype(np.int8)
                inv = np.float32(1) / now[h] if now[h] > 0 else np.float32(0)
                c[h, lo:lo + n] = np.rint(x[h] * inv).astype(np.int8)
            self.scales[t][page] = now

    def append(self, table, sid, pos, k, v):
        """Rows k, v [s, nh * dh] of sequence sid from position pos; what has no page is dropped."""
        s = k.shape[0]
        k, v = k.reshape(s, self.nh, self.dh), v.reshape(s, self.nh, self.dh)
        if not 0 <= sid < table.shape[0] or pos < 0:
            return
        for slot in range(pos // PAGE, (pos + s - 1) // PAGE + 1):
            a, z = max(pos, slot * PAGE), min(pos + s, (slot + 1) * PAGE)
            if slot < table.shape[1] and 0 <= table[sid, slot] < self.n:
                self.store(table[sid, slot], a - slot * PAGE, k[a - pos:z - pos], v[a - pos:z - pos])

    def values(self, t):
        return self.scales[t].astype(np.float64)[:, :, None, None] * self.codes[t]

    def rows(self, table, sid, n):
        """Keys and values of positions 0 .. n-1 in binary64, [nh, n, dh] each."""
        at = np.arange(n)
        pages = table[sid, at // PAGE]
        return [self.values(t)[pages, :, at % PAGE].transpose(1, 0, 2) for t in range(2)]

    # the device's order
    def device_codes(self):
        v = self.codes[1].reshape(self.n, self.nh, 4, 16, self.dh).transpose(0, 1, 2, 4, 3)
        return self.codes[0], np.ascontiguousarray(v)


def attention(q, keys, values, scale):
    """q [nh, dh], keys and values [nkv, n, dh]: binary64 softmax attention, [nh * dh]; no rows: zeros."""
    nh, dh = q.shape
    nkv, n = keys.shape[:2]
    if n == 0:
        return np.zeros(nh * dh), 0.0
    s = np.einsum("kgd,knd->kgn", q.astype(np.float64).reshape(nkv, nh // nkv, dh), keys) * scale
    w = np.exp(s - s.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    return np.einsum("kgn,knd->kgd", w, values).reshape(-1), float(np.abs(s).max())


def select(logits, scores, beams, n_best, done=None, eos=-1):
    """(beams, ids, values in binary64, done) as lists of lists, and all candidates' values in order."""
    x = logits.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
    out = []
    for g in range(len(scores) // beams):
        cand = []
        for j in range(beams):
            row = g * beams + j
            sc = float(scores[row])
            if not sc > -np.inf:
                continue
            if done is not None and done[row]:
                cand.append((-sc, 0.0, j, eos))
                continue
            m = x[row].max()
            if m == -np.inf:
                continue
            lse = m + np.log(np.exp(x[row] - m).sum())
            for w in np.argsort(-x[row], kind="stable")[:n_best]:
                if x[row, w] > -np.inf:
                    cand.append((-(sc + (x[row, w] - lse)), -x[row, w], j, int(w)))
        cand.sort()
        best = [(j, w, -v, int((done is not None and bool(done[g * beams + j])) or (eos >= 0 and w == eos))) for v, _, j, w in cand[:n_best]]
        out.append(best + [(-1, -1, -np.inf, 1)] * (n_best - len(best)))
    return out


def reorder(table, pos, parents, beams, per_group):
    """(table, pos, missing, copies [(row, from, to, rows)])."""
    rows, stride = table.shape
    new, npos = np.full_like(table, -1), np.empty_like(pos)
    missing, copies = np.zeros(rows // beams, np.int32), []
    for g in range(rows // beams):
        lo, hi = g * per_group, (g + 1) * per_group
        n_of = {}
        for i in range(g * beams, (g + 1) * beams):
            p = parents[i] if 0 <= parents[i] < beams else i - g * beams
            src = g * beams + p
            npos[i] = pos[src]
            n_of[i] = min(max(int(pos[src]), 0), stride * PAGE)
            held = -(-n_of[i] // PAGE)
            new[i, :held] = table[src, :held]
        used = {int(p) for i in n_of for p in new[i] if lo <= p < hi}
        free = [p for p in range(lo, hi) if p not in used]
        kept = set()
        for i, n in n_of.items():
            slot = n // PAGE
            if slot >= stride:
                missing[g] += 1
                continue
            page = int(new[i, slot])
            if n % PAGE:
                if lo <= page < hi and page not in kept:
                    kept.add(page)
                    continue
                kept.add(page)
            to = free.pop(0) if free else -1
            missing[g] += to < 0
            new[i, slot] = to
            if n % PAGE and page >= 0 and to >= 0:
                copies.append((i, page, to, (n % PAGE + 15) // 16 * 16))
    return new, npos, missing, copies
