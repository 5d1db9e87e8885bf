"""The bookkeeping of a cache's pages, one entry after the other (numpy and lists; no code shared with the library)."""
import numpy as np

S = 64


def chunks(tokens):
    return -(-tokens // S)


def lengths(p, seqlens):
    return [p.L] * p.B if seqlens is None else [min(max(int(x), 0), p.L) for x in seqlens]


def fresh(p, lens, newlens):
    return [min(p.N if newlens is None else min(max(int(x), 0), p.N), a) for x, a in zip(newlens if newlens is not None else lens, lens)]


def reserve(p, table, refs, pools, seqlens=None, newlens=None):
    """(table, refs, copied, counts); pools are changed."""
    table, refs = [list(map(int, r)) for r in table], list(map(int, refs))
    P, lens = len(refs), lengths(p, seqlens)
    new = fresh(p, lens, newlens)
    begun = {}  # page in use -> the sequences that are about to write to it
    for b in range(p.B):
        start = lens[b] - new[b]
        if new[b] and start % S and 0 <= table[b][start // S] < P:
            begun.setdefault(table[b][start // S], []).append(b)
    copies = set()
    for page, rows in begun.items():
        if refs[page] > 1:
            copies |= set(rows[1:] if len(rows) >= refs[page] else rows)
    needs = []  # (sequence, chunk, page to copy or None)
    for b in range(p.B):
        start = lens[b] - new[b]
        if new[b] and start % S:
            page = table[b][start // S]
            if b in copies:
                needs.append((b, start // S, page))
            elif not 0 <= page < P:
                needs.append((b, start // S, None))
        needs += [(b, c, None) for c in range(chunks(start), chunks(lens[b]))]
    free = [i for i, x in enumerate(refs) if x <= 0]
    found = min(len(needs), len(free))
    copied = np.full((p.B, 2), -1, np.int32)
    if found == len(needs):
        for (b, c, src), dst in zip(needs, free):
            table[b][c], refs[dst] = dst, 1
            if src is not None:
                refs[src] -= 1
                copied[b] = src, dst
                for x in pools:
                    x[dst] = x[src]
    return np.int32(table), np.int32(refs), copied, np.int32([len(needs), found])


def fork(p, parent, table, refs, seqlens=None):
    refs, P, lens, C = list(map(int, refs)), len(refs), lengths(p, seqlens), p.L // S
    out, ends = np.full((len(parent), C), -1, np.int32), []
    for b in range(p.B):
        for c in range(chunks(lens[b])):
            if 0 <= table[b][c] < P:
                refs[table[b][c]] -= 1
    for r, u in enumerate(parent):
        u = int(u)
        ends.append(lens[u] if 0 <= u < p.B else 0)
        for c in range(chunks(ends[-1])):
            out[r, c] = table[u][c]
            if 0 <= table[u][c] < P:
                refs[table[u][c]] += 1
    return out, np.int32(ends), np.int32(refs)


def free(p, keep, table, refs, seqlens=None, pages=None, npages=None):
    table, refs, lens = np.array(table, np.int32), np.array(refs, np.int32), lengths(p, seqlens)
    P, ends = len(refs), []
    for b in range(p.B):
        ends.append(min(lens[b], max(int(keep[b]), 0)))
        gone = list(range(chunks(ends[-1]), chunks(lens[b])))
        give = [int(table[b, c]) for c in gone]
        table[b, gone] = -1
        if pages is not None:
            give += [int(x) for x in pages[b][:len(pages[b]) if npages is None else min(max(int(npages[b]), 0), len(pages[b]))]]
        for x in give:
            if 0 <= x < P:
                refs[x] -= 1
    return table, np.int32(ends), refs


def compact(p, table, refs, pools, seqlens=None):
    """(table, refs, new_page, moved, counts); pools are changed."""
    table, refs, lens = np.array(table, np.int32), [max(0, int(x)) for x in refs], lengths(p, seqlens)
    P = len(refs)
    n = sum(x > 0 for x in refs)
    new_page = [i if x > 0 else -1 for i, x in enumerate(refs)]
    sources, holes = [i for i in range(n, P) if refs[i] > 0], [i for i in range(n) if refs[i] <= 0]
    assert len(sources) == len(holes)
    for src, dst in zip(sources, holes):
        new_page[src], refs[dst], refs[src] = dst, refs[src], 0
        for x in pools:
            x[dst] = x[src]
    for b in range(p.B):
        for c in range(chunks(lens[b])):
            if 0 <= table[b, c] < P:
                table[b, c] = new_page[table[b, c]]
    return table, np.int32(refs), np.int32(new_page), np.int32(sources + [-1] * (P - len(sources))), np.int32([n, len(sources)])
