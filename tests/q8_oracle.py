"""The 8-bit cache's operators in float64 numpy, from their definitions (include/hils.h).

Codes are uint8 arrays (e4m3); k [P, Hkv, 64, d], v [P, Hkv, d, 64], scale [P, Hkv, 2]."""
import numpy as np

S = 64


def _table():
    t = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (e, m) == (15, 7) else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[c] = -x if c & 128 else x
    return t


VALUE = _table()


def encode(x):
    """Nearest code (ties to even) of |x| <= 448; anything not finite is NaN (0x7f)."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    codes = VALUE[:127]  # ascending
    hi = np.clip(np.searchsorted(codes, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dlo, dhi = a - codes[lo], codes[hi] - a
    c = np.where((dlo < dhi) | ((dlo == dhi) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    c = c | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), c, 0x7f).astype(np.uint8)


def scale_for(amax):
    e = -100
    while amax > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def tokens(p, seqlens, newlens, b):
    length = p.L if seqlens is None else min(max(int(seqlens[b]), 0), p.L)
    fresh = min(max(p.N if newlens is None else int(newlens[b]), 0), p.N)
    return length, min(fresh, length)


def append(p, k_new, v_new, k, v, scale, table, seqlens=None, newlens=None):
    """The pools after the call (copies)."""
    k, v, scale = k.copy(), v.copy(), scale.copy()
    for b in range(p.B):
        length, fresh = tokens(p, seqlens, newlens, b)
        start = length - fresh
        for c in range(start // S, -(-length // S)):
            lo, hi = max(start, c * S), min(length, c * S + S)
            if hi <= lo:
                continue
            page = int(table[b, c])
            if not 0 <= page < len(k):
                continue  # no page: dropped
            r0, r1 = lo - c * S, hi - c * S
            for which, new, pool in ((0, k_new, k), (1, v_new, v.transpose(0, 1, 3, 2))):
                for g in range(p.Hkv):
                    x = new[b, g, lo - start:hi - start].astype(np.float64)
                    s = scale_for(np.abs(x[np.isfinite(x)]).max(initial=0.0))
                    if r0:
                        old = float(scale[page, g, which])
                        s = max(s, old)
                        if s != old:
                            pool[page, g, :r0] = encode(VALUE[pool[page, g, :r0]] * (old / s))
                    pool[page, g, r0:r1] = encode(x / s)
                    scale[page, g, which] = s
    return k, v, scale


def landmark(p, lq, k, scale, table, seqlens=None, newlens=None, shared=False):
    """{(page): (k' / scale [Hl, d], b' [Hl])} of the chunks that the call completes."""
    Hl = p.Hl or p.Hq
    out = {}
    for b in range(p.B):
        length, fresh = tokens(p, seqlens, newlens, b)
        first = (length - fresh) // S
        for j, c in enumerate(range(first, length // S)):
            page = int(table[b, c])
            if not 0 <= page < len(k):
                continue  # no page: dropped
            rows, biases = [], []
            for hl in range(Hl):
                g = hl // (Hl // p.Hkv)
                x = VALUE[k[page, g]]
                q = (lq[hl] if shared else lq[b, hl, j]).astype(np.float64)
                s = p.c().scale * float(scale[page, g, 0]) * (x @ q)
                e = np.exp(s - s.max())
                w = e / e.sum()
                rows.append(w @ x)
                biases.append(np.log(e.sum()) - (w * (s - s.max())).sum())
            out[page] = (np.array(rows), np.array(biases))
    return out


def n_candidates(i, W):
    return max(0, i - W + 1) // S


def pieces(W):
    return (W + 62) // 64 + 1


def decode(p, q, k, v, scale, lmk, table, bias=None, q_route=None, seqlens=None, given=None):
    """(out, lse, idx, weights) of every row; `given`: a selection to use (invalid entries ignored)."""
    G, Hl, K, W = p.Hq // p.Hkv, p.Hl or p.Hq, p.topk, p.window
    sc = p.c().scale
    out = np.zeros((p.B, p.Hq, p.N, p.d))
    lse = np.zeros((p.B, p.Hq, p.N))
    idx = np.full((p.B, p.Hkv, p.N, K), -1, np.int32)
    wt = np.zeros((p.B, p.Hkv, p.N, K + pieces(W)))
    P = len(k)
    for b in range(p.B):
        length = p.L if seqlens is None else min(max(int(seqlens[b]), p.N), p.L)
        page = np.clip(table[b], 0, P - 1)
        for n in range(p.N):
            i = length - p.N + n
            nc = n_candidates(i, W)
            for g in range(p.Hkv):
                hs = np.arange(g * G, g * G + G)
                qr = (q if q_route is None else q_route)[b, hs, n].astype(np.float64)
                qq = q[b, hs, n].astype(np.float64)
                hl = hs if Hl == p.Hq else np.full(G, g)
                score = np.zeros((G, nc))
                if nc:
                    lm = VALUE[lmk[page[:nc]][:, hl]] * scale[page[:nc], g, 0].astype(np.float64)[:, None, None]
                    score = sc * np.einsum("chd,hd->hc", lm, qr)
                    if bias is not None:
                        score = score + bias[page[:nc]][:, hl].T
                if given is None:
                    sig = score.max(0) if nc else np.zeros(0)
                    sel = np.sort(np.lexsort((np.arange(nc), -sig))[:K])
                    slots = list(enumerate(sel))
                    idx[b, g, n, :len(sel)] = sel
                else:
                    row = given[b, g, n]
                    slots = [(t, c) for t, c in enumerate(row) if 0 <= c < nc and (t == 0 or c > row[t - 1])]
                    idx[b, g, n] = row

                def attend(c, nk):
                    pg = page[c]
                    ks, vs = scale[pg, g].astype(np.float64)
                    x = sc * (qq @ (VALUE[k[pg, g, :nk]] * ks).T)  # [G, nk]
                    m = x.max(1)
                    e = np.exp(x - m[:, None])
                    with np.errstate(invalid="ignore"):
                        o = e @ (VALUE[v[pg, g, :, :nk]] * vs).T / e.sum(1)[:, None]
                    return m + np.log(e.sum(1)), o

                parts = [(t, score[:, c], attend(c, S)[1]) for t, c in slots]
                for j, c in enumerate(range(nc, i // S + 1)):
                    parts.append((K + j, *attend(c, min(S, i - c * S + 1))))
                z = np.array([x[1] for x in parts])
                m = z.max(0)
                full = m + np.log(np.exp(z - m).sum(0))
                for slot, zz, o in parts:
                    a = np.exp(zz - full)
                    wt[b, g, n, slot] = a.sum()
                    out[b, hs, n] += np.where(a[:, None] > 0, a[:, None] * o, 0.0)
                lse[b, hs, n] = full
    return out, lse, idx, wt


def evict(p, acc, table, seqlens, budget, sink, most, weights=None, idx=None):
    """(acc, table, seqlens, freed, nfreed); sums in float64."""
    nC, K, W = p.L // S, p.topk, p.window
    acc, table = acc.astype(np.float64), table.copy()
    freed, counts, lens = np.full((p.B, most), -1, np.int32), [], []
    for b in range(p.B):
        tokens_ = p.L if seqlens is None else min(max(int(seqlens[b]), 0), p.L)
        length = max(tokens_, p.N)  # the decode call's positions
        if weights is not None:
            for g in range(p.Hkv):
                for n in range(p.N):
                    i = length - p.N + n
                    nc, row = n_candidates(i, W), idx[b, g, n]
                    for t in range(K):
                        if 0 <= row[t] < nc and (t == 0 or row[t] > row[t - 1]):
                            acc[b, row[t]] += weights[b, g, n, t]
                    for c in range(nc, i // S + 1):
                        acc[b, c] += weights[b, g, n, K + c - nc]
        last = n_candidates(tokens_ - 1, W)
        able = list(range(sink, last))
        count = min(max(0, last - budget), len(able), most)
        gone = sorted(sorted(able, key=lambda c: (np.isnan(acc[b, c]), acc[b, c], c))[:count])
        kept = [c for c in range(nC) if c not in set(gone)]
        freed[b, :count] = table[b, gone]
        acc[b] = np.concatenate([acc[b, kept], np.zeros(count)])
        table[b] = np.concatenate([table[b, kept], np.full(count, -1)])
        counts.append(count)
        lens.append(tokens_ - S * count)
    return acc, table, np.array(lens, np.int32), freed, np.array(counts, np.int32)
