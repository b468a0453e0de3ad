"""Plain 64-bit oracle of the answer's operators: tables of new rows, attention over the paged context, the next token.

Test infrastructure only: numpy loops written from the definitions, sharing no code with the GPU path."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
OK, NO_PAGES, TABLE_FULL, ORDER, NO_ROWS = range(5)


def _pages(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def extend_segments(segs, n_new, tab_cap, req_seg_off, free_blocks, block_tab, n_blocks, max_rows):
    """Returns (segs, block_tab, cu_q, q_pos, slot_map, row_req, last_row, status, counts)."""
    segs, tab = np.array(segs, dtype=np.int64), np.array(block_tab, dtype=np.int64)
    n_req = len(req_seg_off) - 1
    status = np.zeros(n_req, np.int64)
    spans = [range(int(req_seg_off[r]), int(req_seg_off[r + 1])) for r in range(n_req)]
    old = [max(int(v), 0) for v in segs[:, 3]]
    add = [max(int(v), 0) for v in n_new]
    wish_pages = wish_rows = 0
    for r, span in enumerate(spans):
        pages = sum(_pages(old[s] + add[s]) - _pages(old[s]) for s in span)
        rows = sum(add[s] for s in span)
        full = any(add[s] and (segs[s, 4] < 0 or _pages(old[s] + add[s]) > tab_cap[s] or segs[s, 4] + _pages(old[s] + add[s]) > len(tab)) for s in span)
        if full or sum(old[s] + add[s] for s in span) >= 2 ** 31:
            status[r] = TABLE_FULL
        elif any(add[s] and any(old[t] for t in span if t > s) for s in span):
            status[r] = ORDER
        else:
            wish_pages, wish_rows = wish_pages + pages, wish_rows + rows
            if pages and wish_pages > len(free_blocks):
                status[r] = NO_PAGES
            elif rows and wish_rows > max_rows:
                status[r] = NO_ROWS
    cu, pos, slot, row_req, last = [0], [], [], [], []
    token = taken = 0
    for r, span in enumerate(spans):
        start = 0
        for s in span:
            n = add[s] if status[r] == OK else 0
            for b in range(_pages(old[s]), _pages(old[s] + n)):
                tab[segs[s, 4] + b] = free_blocks[taken]
                taken += 1
            segs[s] = [r, segs[s, 1], start, old[s] + n, segs[s, 4], n, token, len(pos)]
            for t in range(old[s], old[s] + n):
                page = int(tab[segs[s, 4] + t // BLOCK])
                pos.append(start + t)
                slot.append(page * BLOCK + t % BLOCK if 0 <= page < n_blocks else -1)
                row_req.append(r)
            start += old[s] + n
            token += old[s] + n
        last.append(len(pos) - 1 if len(pos) > cu[-1] else -1)
        cu.append(len(pos))
    n = len(pos)
    fill = lambda v, w: np.array(v + [w] * (max_rows - n), dtype=np.int32)
    return (segs.astype(np.int32), tab.astype(np.int32), np.array(cu, np.int32), fill(pos, 0), fill(slot, -1), fill(row_req, -1),
            np.array(last, np.int32), status.astype(np.int32), np.array([n, taken, int((status != OK).sum()), token], np.int32))


def rotate(x, pos, theta):
    """x [rows, heads, d] at positions pos."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    a = np.asarray(pos, np.float64)[:, None] * theta ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    return np.concatenate([x[..., :half] * c - x[..., half:] * s, x[..., half:] * c + x[..., :half] * s], -1)


def paged_context(k_pool, v_pool, v_of, block_tab, segs, span):
    """Positions, keys [n, Hkv, d] and values of the segments `span`; pages outside the pool are left out.  v_of(block) -> [Hkv, d, 16]."""
    pos, keys, values = [], [], []
    for s in span:
        _, _, start, n, tab = (int(v) for v in segs[s][:5])
        for b in range(_pages(n)):
            page, m = int(block_tab[tab + b]), min(BLOCK, n - b * BLOCK)
            if not 0 <= page < len(k_pool):
                continue
            pos.append(start + b * BLOCK + np.arange(m))
            keys.append(np.moveaxis(np.asarray(k_pool[page], np.float64), 1, 0)[:m])
            values.append(np.moveaxis(np.asarray(v_of(page), np.float64), 2, 0)[:m])
    if not pos:
        h, d = k_pool.shape[1], k_pool.shape[3]
        return np.zeros(0, np.int64), np.zeros((0, h, d)), np.zeros((0, h, d))
    return np.concatenate(pos), np.concatenate(keys), np.concatenate(values)


def attend(q, q_pos, pos, keys, values, theta, half_step):
    """(out, lse, bound of out, bound of lse) of rows q [n, Hq, d] over a context.  The bounds are what a computation may be off that rounds
    the turned query, the weights and the output once each to a type of relative half step `half_step` and otherwise works in
    32 bits: with u = 2^-24, a logit is off by at most  e = (half_step + (d + 8) u) sum|q k| / sqrt d + 4 u |z|, a weight by
    2 max e + half_step + 8 u relatively, a sum of n terms by n u."""
    q = rotate(q, q_pos, theta)
    n, hq, d = q.shape
    group, u = hq // keys.shape[1], 2.0 ** -24
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    out_bound, lse_bound = np.zeros((n, hq, d)), np.zeros((n, hq))
    for i in range(n):
        seen = pos <= q_pos[i]
        if not seen.any():
            continue
        k, v = keys[seen], values[seen]
        for h in range(hq):
            kh, vh = k[:, h // group], v[:, h // group]
            z = kh @ q[i, h] / math.sqrt(d)
            e = ((half_step + (d + 8) * u) * (np.abs(kh) @ np.abs(q[i, h])) / math.sqrt(d) + 4 * u * (np.abs(z) + np.abs(z).max())).max()
            w = np.exp(z - z.max())
            total = w.sum()
            p = w / total
            out[i, h] = p @ vh
            lse[i, h] = z.max() + math.log(total)
            rel = math.expm1(2 * e) + half_step + (2 * len(z) + 16) * u
            out_bound[i, h] = half_step * np.abs(out[i, h]) + rel * (p @ np.abs(vh)) + 1e-30
            lse_bound[i, h] = e + (len(z) + 16) * u + 4 * u * abs(lse[i, h])
    return out, lse, out_bound, lse_bound


def sample(z, temperature, top_k, top_p, min_p, u):
    """(token, logprob, n_kept) of one row of logits."""
    z = np.array(z, np.float64)
    z[np.isnan(z)] = -np.inf
    rank = np.lexsort((np.arange(len(z)), -z))
    rank = rank[z[rank] > -np.inf]
    if len(rank) == 0:
        return -1, -math.inf, 0
    if not temperature > 0:
        return int(rank[0]), 0.0, 1
    top = z[rank[0]]
    w = np.where(z[rank] == top, 1.0, 0.0) if np.isposinf(top) else np.exp((z[rank] - top) / temperature)
    n = top_k if 0 < top_k < len(w) else len(w)
    if top_p < 1:
        mass = np.cumsum(w[:n])
        n = 1 + int((mass[:-1] < max(top_p, 0.0) * mass[-1]).sum())
    if min_p > 0:
        n = max(1, min(n, int((w >= min_p).sum())))
    at = np.argsort(rank[:n])
    sums = np.cumsum(w[:n][at])
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    i = int(np.searchsorted(sums, u * sums[-1], side="right"))
    return int(rank[at[i]]), math.log(w[at[i]] / sums[-1]), n
