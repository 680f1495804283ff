"""Reordering of page tables by the definition in include/fg.h, for rows of any lengths: a begun page that a row of the group also
holds as a full page (a beam taken back to a shorter length, a fork from an earlier position) is not the row's to write to."""
import numpy as np

PAGE = 64


def reorder(table, pos, parents, beams, per_group):
    """(table, pos, missing, copies [(row, from, to, rows)])."""
    rows, stride = table.shape
    local = np.arange(rows) % beams
    par = np.where((parents >= 0) & (parents < beams), parents, local) + np.arange(rows) - local
    npos = pos[par]
    n = np.clip(npos.astype(np.int64), 0, stride * PAGE)
    new = np.where(np.arange(stride) < ((n + PAGE - 1) // PAGE)[:, None], table[par], -1).astype(table.dtype)
    missing, copies = np.zeros(rows // beams, np.int32), []
    for g in range(rows // beams):
        mine = range(g * beams, (g + 1) * beams)
        own = range(g * per_group, (g + 1) * per_group)
        full = {int(p) for i in mine for p in new[i, :n[i] // PAGE]}
        held = {int(p) for i in mine for p in new[i]}
        free = iter([p for p in own if p not in held])
        given = set()
        for i in mine:
            at, begun = int(n[i]) // PAGE, int(n[i]) % PAGE
            if at == stride:
                missing[g] += 1
                continue
            page = int(new[i, at])
            if begun and page in own and page not in full and page not in given:
                given.add(page)
                continue
            to = next(free, -1)
            new[i, at] = to
            missing[g] += to < 0
            if begun and page >= 0 and to >= 0:
                copies.append((i, page, to, -(-begun // 16) * 16))
    return new, npos, missing, copies


def tree(r, groups, beams, stride, per_group):
    """Tables as forks leave them: rows that share the pages of a random number of positions, taken back to random lengths."""
    table = np.full((groups * beams, stride), -1, np.int32)
    pos = np.zeros(groups * beams, np.int32)
    for g in range(groups):
        ids = list(g * per_group + r.permutation(per_group))
        for i in range(g * beams, (g + 1) * beams):
            pos[i] = r.integers(0, (stride - 1) * PAGE + 1)
            used = -(-int(pos[i]) // PAGE)
            shared = 0
            if i > g * beams:
                k = int(r.integers(g * beams, i))
                shared = min(int(r.integers(0, stride)), used, -(-int(pos[k]) // PAGE))
                table[i, :shared] = table[k, :shared]
            for c in range(shared, used):
                table[i, c] = ids.pop()
    return table, pos
