"""Paged key-value cache in plain numpy (fp64), from the definitions in include/alr.h."""

import numpy as np


def plan(length, add, pool, pool_used, table, page, T):
    """One sequence after the other; returns a dict of the outputs, table and pool included."""
    S, cols = table.shape
    table, pool, length = table.copy(), [int(p) for p in pool], [int(n) for n in length]
    pages = lambda n: -(-n // page)  # noqa: E731
    back = [int(table[s, j]) for s in range(S) if add[s] < 0 for j in range(pages(length[s]))]
    used = int(pool_used) - len(back)
    for i, p in enumerate(back):
        pool[used + i] = p
    o = dict(slot=np.full(T, -1), tok_seq=np.full(T, -1), tok_len=np.zeros(T, int),
             start=np.zeros(S + 1, int), n_refused=0)
    row, asked, taken, free = 0, 0, 0, len(pool) - used
    for s in range(S):
        n, a = length[s], int(add[s])
        o["start"][s] = row
        if a < 0:
            length[s] = 0
            continue
        need = pages(n + a) - pages(n)
        ok = n + a <= cols * page and row + a <= T
        if ok:
            asked += need
            ok = need == 0 or asked <= free
        if not ok:
            o["n_refused"] += 1
        else:
            for j in range(need):
                table[s, pages(n) + j] = pool[used + asked - need + j]
            taken = asked if need else taken
            for i in range(a):
                o["slot"][row + i] = table[s, (n + i) // page] * page + (n + i) % page
                o["tok_seq"][row + i], o["tok_len"][row + i] = s, n + i + 1
            length[s] = n + a
        row += a
    o["start"][S] = row
    o.update(len=np.array(length, int), table=table, pool=np.array(pool, int), pool_used=used + taken)
    return o


def tokens_of(table, n_pages, page, seq, length):
    """(page, position) of the tokens that a row reads, as two arrays."""
    n_seq, cols = table.shape
    if not 0 <= seq < n_seq:
        length = 0
    t = np.arange(min(max(int(length), 0), cols * page))
    pg = table[seq if 0 <= seq < n_seq else 0, t // page].astype(int)
    there = (pg >= 0) & (pg < n_pages)
    return pg[there], (t % page)[there]


def attention(Q, K, V, table, parts, scale):
    """Q [N, H, D], K, V [n_pages, page, heads, D] fp64; parts: (seq, len) arrays by row.  Returns out,
    lse and for error bounds: size (sum of the weights times |v|), reach (largest sum of |q k| scale
    over the tokens that have a weight), n (tokens of the row)."""
    N, H, D = Q.shape
    n_pages, page, heads, _ = K.shape
    g = H // heads
    out, size = np.zeros((N, H, D)), np.zeros((N, H, D))
    lse, reach, n = np.full((N, H), -np.inf), np.zeros((N, H)), np.zeros(N, int)
    for r in range(N):
        at = [tokens_of(table, n_pages, page, int(seq[r]), length[r]) for seq, length in parts]
        pg, pos = (np.concatenate([a[i] for a in at]) for i in range(2))
        n[r] = len(pg)
        if not n[r]:
            continue
        k, v = K[pg, pos], V[pg, pos]                        # [tokens, heads, D]
        for h in range(H):
            kh, vh = k[:, h // g], v[:, h // g]
            x = scale * (kh @ Q[r, h])
            m = x.max()
            if m == -np.inf:
                continue
            e = np.exp(x - m)
            reach[r, h] = abs(scale) * np.max(np.abs(kh[e > 0]) @ np.abs(Q[r, h]))
            out[r, h], size[r, h] = e @ vh / e.sum(), e @ np.abs(vh) / e.sum()
            lse[r, h] = m + np.log(e.sum())
    return out, lse, size, reach, n
