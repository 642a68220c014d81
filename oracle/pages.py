"""CPU oracle of the paged K/V cache (numpy; float64 where numbers are
computed), written from the definitions: the stack of free pages is a Python
list that requests pop from and push to in turn, attention is a softmax over
the tokens a row sees, gathered one by one from their pages."""
from __future__ import annotations

import numpy as np

FLAG_OUT_CAPACITY, FLAG_BAD_PAGE, FLAG_NO_PAGES = 8, 16, 32


def page_tables(page_size, cu_new, seq_len, free_pages, free_count, block_table, n_new):
    """-> (block_table, slot_map, seq_len_out, free_count_out, flags)"""
    n_pages, B = len(free_pages), len(seq_len)
    table = np.array(block_table, dtype=np.int64)
    stack = list(free_pages[:min(free_count, n_pages)])
    slots = np.full(n_new, -1, dtype=np.int64)
    lens = np.array(seq_len, dtype=np.int64)
    flags = np.zeros(B, dtype=np.int64)
    short = False                      # a request before went without: so does every later one in need
    for b in range(B):
        L, n = int(seq_len[b]), int(cu_new[b + 1] - cu_new[b])
        held, want = -(-L // page_size), -(-(L + n) // page_size)
        if want > table.shape[1] or cu_new[b + 1] > n_new:
            flags[b] |= FLAG_NO_PAGES
            continue
        if want > held and (short or want - held > len(stack)):
            short = True
            flags[b] |= FLAG_NO_PAGES
            continue
        for p in range(held, want):
            table[b, p] = stack.pop()
        for i in range(n):
            page = table[b, (L + i) // page_size]
            if 0 <= page < n_pages:
                slots[cu_new[b] + i] = page * page_size + (L + i) % page_size
            else:
                flags[b] |= FLAG_BAD_PAGE
        lens[b] = L + n
    return table, slots, lens, len(stack), flags


def page_trim(page_size, keep_len, seq_len, block_table, free_pages, free_count):
    """-> (free_pages, seq_len_out, free_count_out, flags)"""
    stack = [int(x) for x in free_pages[:free_count]]
    lens, flags = np.array(seq_len, dtype=np.int64), np.zeros(len(seq_len), dtype=np.int64)
    for b in range(len(seq_len)):
        keep = min(int(keep_len[b]), int(seq_len[b]))
        for p in range(-(-keep // page_size), -(-int(seq_len[b]) // page_size)):
            if len(stack) < len(free_pages):
                stack.append(int(block_table[b, p]))
            else:
                flags[b] |= FLAG_OUT_CAPACITY
        lens[b] = keep
    out = np.array(free_pages, dtype=np.int64)
    out[:len(stack)] = stack
    return out, lens, len(stack), flags


def page_store(pages, rows, slot_map, keep_idx=None):
    """pages [n_pages, Hkv, page_size, d] with the rows [n, Hkv, d] in their slots"""
    out = np.array(pages)
    n_pages, _, ps, _ = out.shape
    for r, s in enumerate(slot_map):
        j = r if keep_idx is None else int(keep_idx[r])
        if 0 <= s < n_pages * ps and 0 <= j < len(rows):
            out[s // ps, :, s % ps] = rows[j]
    return out


def gather(pages, row, length):
    """Tokens [length, Hkv, d] of one sequence; pages outside the pool are zeros."""
    n_pages, Hkv, ps, d = pages.shape
    out = np.zeros((length, Hkv, d), dtype=np.float64)
    for t in range(length):
        p = int(row[t // ps])
        if 0 <= p < n_pages:
            out[t] = pages[p, :, t % ps]
    return out


def page_attention(k_pages, v_pages, q, cu_q, kv_len, block_table, scale):
    """-> (out [N, Hq, d], lse [Hq, N], bound): float64; rows of no sequence are
    NaN.  bound holds, for every row, sum p |v| ([N, Hq, d]) and the largest
    c sum |q k| over the row's keys ([Hq, N]): what the rounding of p and of the
    products is relative to."""
    N, Hq, d = q.shape
    Hkv, ps = k_pages.shape[1], k_pages.shape[2]
    G = Hq // Hkv
    out = np.full((N, Hq, d), np.nan)
    lse = np.full((Hq, N), np.nan)
    weight = np.zeros((N, Hq, d))
    reach = np.zeros((Hq, N))
    with np.errstate(all="ignore"):
        for b in range(len(kv_len)):
            n = int(cu_q[b + 1] - cu_q[b])
            L = max(0, min(int(kv_len[b]), block_table.shape[1] * ps))
            k, v = gather(k_pages, block_table[b], L), gather(v_pages, block_table[b], L)
            for t in range(n):
                seen = min(L, int(kv_len[b]) - n + t + 1)
                r = int(cu_q[b]) + t
                for h in range(Hq):
                    if seen <= 0:
                        out[r, h], lse[h, r] = 0.0, -np.inf
                        continue
                    kk, vv, qq = k[:seen, h // G], v[:seen, h // G], q[r, h].astype(np.float64)
                    z = scale * (kk @ qq)
                    top = z.max()
                    e = np.exp(z - top)
                    total = e.sum()
                    out[r, h] = (e / total) @ vv
                    lse[h, r] = top + np.log(total)
                    weight[r, h] = (e / total) @ np.abs(vv)
                    reach[h, r] = (scale * (np.abs(kk) @ np.abs(qq))).max()
    return out, lse, (weight, reach)
