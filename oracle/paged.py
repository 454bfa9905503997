"""Plain numpy forms of the paged cache's operators (include/fathom.h), one request at a time, sums in 64 bits."""
import numpy as np


def pages_of(n, page):
    return (int(n) + page - 1) // page


def paged_map(n_old, n, page, table, ring, state, T, H):
    """(table, ring, slots, start, n_now, n_unit, state_out, short, bad_n) as fathom_paged_map defines them, for page
    numbers inside the pool and a state that can be."""
    table, ring = table.copy(), ring.copy()
    S, L = table.shape
    P, head, count = len(ring), int(state[0]), int(state[1])
    free = [(head + i) % P for i in range(count)]
    start, slots, n_now = np.zeros(S + 1, np.int64), np.full(T, -1, np.int64), np.zeros(S, np.int64)
    taken = popped = at = 0
    short = bad_n = False
    returned = []
    for s in range(S):
        a, b = int(n_old[s]), int(n[s])
        start[s] = at
        inside = 0 <= a <= L * page
        n_now[s] = a if inside else 0
        if not inside or not 0 <= b <= L * page:
            bad_n = True
            continue
        new, pa, pb = max(b - a, 0), pages_of(a, page), pages_of(b, page)
        row, at = at, at + new
        need = max(pb - pa, 0)
        taken += need
        returned += [table[s, j] for j in range(pb, pa)]
        if new and at > T:
            bad_n = True
        elif need and taken > count:
            short = True
        else:
            n_now[s] = b
            for j in range(need):
                table[s, pa + j] = ring[free[popped]]
                popped += 1
            for i in range(new):
                slots[row + i] = int(table[s, (a + i) // page]) * page + (a + i) % page
    start[S] = at
    for i, p in enumerate(returned):
        ring[(head + count + i) % P] = p
    state_out = np.array([(head + popped) % P, count - popped + len(returned)], np.int64)
    return table, ring, slots, start, n_now, np.repeat(n_now, H), state_out, short, bad_n


def paged_rows(pages, table, s, h, n):
    """Rows [n][D] of head h of request s."""
    page = pages.shape[2]
    return np.concatenate([pages[table[s, j], h] for j in range(pages_of(n, page))] or [np.zeros((0, pages.shape[3]))])[:n]


def paged_attn(q, K, V, n, G, sm_scale, softcap=0.0, slopes=None, prefix=None, first=None):
    """One request and KV head: q [new][G][D], K and V [n][D] in 64 bits -> (out [new][G][D], scale of the sum
    sum_j p_j |V_j| [new][G][D], largest |q||K| sum of a score [new][G]).  prefix: a length or None; first [new] or None;
    slopes [G] or None.  Rows that a token does not see do not enter its result."""
    new, D = q.shape[0], q.shape[2]
    out, mag = np.zeros((new, G, D)), np.zeros((new, G, D))
    top = np.zeros((new, G))
    for i in range(new):
        p = n - new + i
        lo = 0 if first is None else max(int(first[i]), 0)
        hi = p + 1 if prefix is None else max(p + 1, min(int(prefix), n))
        if lo >= hi:
            continue
        j = np.arange(lo, hi)
        for g in range(G):
            z = (K[lo:hi] @ q[i, g]) * sm_scale
            top[i, g] = (np.abs(K[lo:hi]) @ np.abs(q[i, g])).max() * abs(sm_scale)
            if softcap:
                z = softcap * np.tanh(z / softcap)
            if slopes is not None:
                z = z - slopes[g] * np.abs(p - j)
            w = np.exp(z - z.max())
            w /= w.sum()
            out[i, g] = (w[:, None] * V[lo:hi]).sum(0)
            mag[i, g] = (w[:, None] * np.abs(V[lo:hi])).sum(0)
    return out, mag, top
