"""The operators around the indexer in plain numpy, 64 bits: block tables and slot maps, rows written into a cache, and
attention over the positions that a query sees or is given.  Test infrastructure; shares no code with the library."""
from __future__ import annotations

import numpy as np


def page_tables(ctx_len, new_len, block_table, page, free_pages, rows, s_max=0):
    """What hisa_page_tables writes, sequence by sequence; block_table is copied, not changed."""
    table = np.array(block_table, dtype=np.int64)
    n_seq, max_pages = table.shape
    cap = max_pages * page
    seq_len, q_start, page_start = [], [0], [0]
    q_seq, q_pos = np.zeros(rows, np.int64), np.full(rows, -1, np.int64)
    slots, key_rows = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    for n in range(n_seq):
        ctx, new = max(0, int(ctx_len[n])), max(0, int(new_len[n]))
        end = min(ctx + new, cap)
        seq_len.append(end)
        had, need = -(-min(ctx, cap) // page), -(-end // page)
        for j in range(had, need):
            f = page_start[n] + j - had
            table[n, j] = free_pages[f] if f < len(free_pages) else -1
        page_start.append(page_start[n] + need - had)
        q_start.append(min(rows, q_start[n] + new))
        for t in range(q_start[n], q_start[n + 1]):
            pos = min(ctx + t - q_start[n], 2 ** 31 - 1)
            q_seq[t], q_pos[t] = n, pos
            if pos < end and table[n, pos // page] >= 0:
                slots[t] = table[n, pos // page] * page + pos % page
            if pos < s_max:
                key_rows[t] = n * s_max + pos
    return dict(seq_len=np.array(seq_len), q_start=np.array(q_start), page_start=np.array(page_start), q_seq=q_seq,
                q_pos=q_pos, slots=slots, key_rows=key_rows, block_table=table)


def attend(q, k, v, scale):
    """q [G, d], k, v [n, d]: softmax(scale * q k^T) v, its log-sum-exp, and sum p |v| / sum p (what rounding errors of
    the weights scale with).  n == 0: zeros and -inf."""
    if k.shape[0] == 0:
        z = np.zeros((q.shape[0], v.shape[1]))
        return z, np.full(q.shape[0], -np.inf), z
    x = scale * (q @ k.T)
    top = x.max(axis=1, keepdims=True)
    p = np.exp(x - top)
    total = p.sum(axis=1, keepdims=True)
    return p @ v / total, (top + np.log(total))[:, 0], p @ np.abs(v) / total


def gather(rows, block_table, positions, page, n_pages, length):
    """Rows [n, H_kv, d] (and which of the positions there were) of a cache given as [n_pages * page, H_kv, d]."""
    positions = np.asarray(positions, dtype=np.int64)
    positions = positions[(positions >= 0) & (positions < length)]
    pages = block_table[positions // page]
    ok = (pages >= 0) & (pages < n_pages)
    return rows[pages[ok] * page + positions[ok] % page]


def attention(q, k, v, block_table, seq_len, page, seq_of, positions_of, scale):
    """q [T, H, d], k, v [n_pages * page, H_kv, d], all float64; seq_of(t) -> sequence or None (nobody's row),
    positions_of(t) -> positions in any order.  Returns out, lse, mag [T, H, .] with NaN in nobody's rows."""
    T, H, d = q.shape
    H_kv = k.shape[1]
    G = H // H_kv
    n_pages = k.shape[0] // page
    cap = block_table.shape[1] * page
    out, mag, lse = np.full((T, H, d), np.nan), np.full((T, H, d), np.nan), np.full((T, H), np.nan)
    for t in range(T):
        n = seq_of(t)
        if n is None:
            continue
        length = min(int(seq_len[n]), cap) if 0 <= n < len(seq_len) else 0
        row = block_table[n] if length else None
        kk = gather(k, row, positions_of(t), page, n_pages, length) if length > 0 else k[:0]
        vv = gather(v, row, positions_of(t), page, n_pages, length) if length > 0 else v[:0]
        for h in range(H_kv):
            s = slice(h * G, (h + 1) * G)
            out[t, s], lse[t, s], mag[t, s] = attend(q[t, s], kk[:, h], vv[:, h], scale)
    return out, lse, mag
