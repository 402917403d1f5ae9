"""Plain implementations of the paged-cache operators, in numpy and 64 bits, one
sequence and one row at a time."""
import numpy as np


def tree_rows(table, length, held, page, start, parent, T, words, shift=None, n_pages=None):
    """pos, slot [T] and mask [T][words] of vsr_tree_rows."""
    pos, slot = np.zeros(T, np.int32), np.full(T, -1, np.int32)
    mask = np.zeros((T, words), np.uint32)
    for s in range(len(length)):
        b, e = (s, s + 1) if start is None else (int(start[s]), int(start[s + 1]))
        h = min(max(int(held[s]), 0), table.shape[1])
        n = min(max(int(length[s]), 0), h * page)
        depth = {}
        for j in range(e - b):
            up = j - 1 if parent is None else int(parent[b + j])
            if not 0 <= up < j:
                up = -1
            depth[j] = depth[up] + 1 if up >= 0 else 0
            pos[b + j] = n + depth[j] + (0 if shift is None else int(shift[s]))
            if up >= 0:
                mask[b + j] = mask[b + up]
            if j // 32 < words:
                mask[b + j, j // 32] |= np.uint32(1 << j % 32)
            at = n + j
            if at < h * page:
                p = int(table[s, at // page])
                if n_pages is None or 0 <= p < n_pages:
                    slot[b + j] = p * page + at % page
    return pos, slot, mask


def attention(q, k, v, table, length, held, page, start, mask, scale):
    """out [T][Hq][hd], lse [T][Hq], and what bounds an error: the sums of p |v| and the
    largest sum of |q k| a row has; all float64. Rows of no sequence: NaN. k, v:
    [slots][Hk][hd]."""
    T, hq, hd = q.shape
    G = hq // k.shape[1]
    out, lse = np.full((T, hq, hd), np.nan), np.full((T, hq), np.nan)
    mass, size = np.zeros((T, hq, hd)), np.zeros((T, hq))
    n_pages = k.shape[0] // page
    for s in range(len(length)):
        b, e = (s, s + 1) if start is None else (int(start[s]), int(start[s + 1]))
        room = min(max(int(held[s]), 0), table.shape[1]) * page
        n = min(max(int(length[s]), 0), room)
        keys = min(n + e - b, room)
        at = np.arange(keys)
        pages = table[s, at // page].astype(np.int64)
        pages = np.where((pages >= 0) & (pages < n_pages), pages, 0)
        ks, vs = k[pages * page + at % page], v[pages * page + at % page]
        for j in range(e - b):
            d = at - n
            if mask is None:
                seen = d <= j
            else:
                w = np.clip(d, 0, None)
                bit = np.zeros(keys, bool)
                ok = (d >= 0) & (w // 32 < mask.shape[1])
                bit[ok] = mask[b + j, w[ok] // 32] >> (w[ok] % 32).astype(np.uint32) & 1
                seen = (d < 0) | bit
            if not seen.any():
                out[b + j], lse[b + j] = 0, -np.inf
                continue
            for h in range(hq):
                kk, vv = ks[seen, h // G].astype(np.float64), vs[seen, h // G].astype(np.float64)
                qq = q[b + j, h].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    x = kk @ qq * scale
                    m = x.max()
                    p = np.exp(x - m)
                    lse[b + j, h] = m + np.log(p.sum())
                    p /= p.sum()
                    out[b + j, h] = p @ vv
                    mass[b + j, h] = p @ np.abs(vv)
                    size[b + j, h] = abs(scale) * (np.abs(kk) @ np.abs(qq)).max()
    return out, lse, mass, size


def pages_update(table, length, held, refs, page, source, room, k, v):
    """vsr_pages_update in place, one sequence after the other; returns ok. k, v:
    [layers][slots][...]."""
    n, most = table.shape
    was = [list(table[s, :held[s]]) for s in range(n)]
    lens = [int(x) for x in length]
    src = [d if source is None else int(source[d]) for d in range(n)]
    src = [d if not -1 <= s < n else s for d, s in enumerate(src)]
    heir = {s: s if src[s] == s else min([d for d in range(n) if src[d] == s], default=None)
            for s in range(n)}
    mine, copy = [], []
    for d, s in enumerate(src):
        if s == d:
            mine.append(was[d])
            copy.append(None)
            continue
        for p in was[d]:
            refs[p] -= 1
        if s < 0:
            mine.append([])
            copy.append(None)
            length[d] = 0
            continue
        full, part = divmod(lens[s], page)
        pages = was[s][:full + (part > 0)]
        table[d, :len(pages)] = pages
        length[d] = lens[s]
        copy.append(pages.pop() if part and heir[s] != d else None)
        for p in pages:
            refs[p] += 1
        mine.append(pages)
    free = [p for p in range(len(refs)) if refs[p] == 0]
    ok, before = np.zeros(n, np.int32), 0
    for d in range(n):
        have = len(mine[d]) + (copy[d] is not None)
        want = -(-(int(length[d]) + (0 if room is None else max(0, int(room[d])))) // page)
        need = (copy[d] is not None) + (max(0, want - have) if want <= most else 0)
        before += need
        served = need == 0 or before <= len(free)
        ok[d] = served and want <= most
        held[d] = len(mine[d]) + (need if served else 0)
        if served:
            new = free[before - need:before]
            at = len(mine[d])
            table[d, at:at + need] = new
            for p in new:
                refs[p] = 1
            if copy[d] is not None:
                r = np.arange(int(length[d]) % page)
                for x in (k, v):
                    x[:, new[0] * page + r] = x[:, copy[d] * page + r]
        elif copy[d] is not None:
            length[d] = int(length[d]) // page * page
    return ok


def pages_keep(table, length, held, refs, page, kept, n_kept, k, v, release):
    """vsr_pages_keep in place; returns the new lengths."""
    new = length.copy()
    for s in range(len(length)):
        n = kept.shape[1] if n_kept is None else min(max(int(n_kept[s]), 0), kept.shape[1])
        room, last, i = int(held[s]) * page - int(length[s]), -1, 0
        while i < n and last < kept[s, i] < room:
            last = int(kept[s, i])
            x, y = int(length[s]) + last, int(length[s]) + i
            x, y = (int(table[s, p // page]) * page + p % page for p in (x, y))
            k[:, y], v[:, y] = k[:, x].copy(), v[:, x].copy()
            i += 1
        new[s] += i
        if release:
            left = -(-int(new[s]) // page)
            for c in range(left, int(held[s])):
                refs[table[s, c]] -= 1
            held[s] = left
    return new
