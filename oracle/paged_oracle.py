"""fp64 CPU oracle of the paged K/V cache: block tables, slots, rows into pages, attention of one new token per request.

TEST INFRASTRUCTURE ONLY, like pafu_oracle: request by request and token by token from the definitions, in float64 and
Python integers, with no code of the library.  Pages are arrays [n_pages, page_size, N_kv, D].
"""

from __future__ import annotations

import math

import numpy as np

INT_MAX = 2 ** 31 - 1


def paged_tables(kv_len, new_len, free_pages, page_size, block_table, max_slots, free_start=0):
    """-> (block_table, slots, row_start, kv_len_out, free_end): pages in the order of the requests, from free_start on."""
    table = np.array(block_table, dtype=np.int64, copy=True)
    at, row = max(int(free_start), 0), 0
    slots, row_start, out = [], [0], []
    for b, (kv, new) in enumerate(zip(kv_len, new_len)):
        kv, new = max(int(kv), 0), max(int(new), 0)
        have, want = -(-kv // page_size), -(-(kv + new) // page_size)
        taken = {}
        for col in range(have, want):
            taken[col] = int(free_pages[at]) if at < len(free_pages) else -1
            if col < table.shape[1]:
                table[b, col] = taken[col]
            at += 1
        for j in range(kv, kv + new):
            slots.append(_slot(table, b, j, page_size))
        row += new
        row_start.append(min(row, INT_MAX))
        out.append(min(kv + new, INT_MAX))
    return table, _fill(slots, max_slots), np.array(row_start), np.array(out), min(at, INT_MAX)


def paged_slots(block_table, start, count, page_size, max_slots):
    """-> (slots, row_start) of tokens that have their pages."""
    slots, row_start = [], [0]
    for b, (s, n) in enumerate(zip(start, count)):
        s, n = max(int(s), 0), max(int(n), 0)
        slots += [_slot(block_table, b, j, page_size) for j in range(s, s + n)]
        row_start.append(row_start[-1] + n)
    return _fill(slots, max_slots), np.array(row_start)


def _slot(table, b, token, page_size):
    col = token // page_size
    page = int(table[b][col]) if col < table.shape[1] else -1
    slot = page * page_size + token % page_size
    return slot if page >= 0 and (page + 1) * page_size - 1 <= INT_MAX else -1


def _fill(slots, max_slots):
    return np.array((slots + [-1] * max(0, max_slots - len(slots)))[:max_slots], dtype=np.int64)


def paged_append(pages, rows, slots):
    """A copy of `pages` (values or codes) with rows[t] at slots[t]; slots outside the pool are left out."""
    out = np.array(pages, copy=True)
    n_pages, page_size = out.shape[:2]
    for row, slot in zip(rows, slots):
        if 0 <= slot < n_pages * page_size:
            out[slot // page_size, slot % page_size] = row
    return out


def visible_tokens(kv_len, n_pinned, window, most=INT_MAX):
    """Tokens of a request that its new token attends to: all, or the last `window` and the first `n_pinned`; of these the
    ones below `most` (what the table holds)."""
    return [j for j in range(min(max(int(kv_len), 0), most)) if window <= 0 or j < n_pinned or j >= kv_len - window]


def paged_attention(Q, K_pages, V_pages, block_table, kv_len, scale=None, n_pinned=0, window=0):
    """O [B, N, D] in float64; tokens on pages outside the pool or the table are not visible, empty rows are 0."""
    Q = np.asarray(Q, dtype=np.float64)
    B, N, D = Q.shape
    n_pages, page_size, N_kv = K_pages.shape[:3]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    O = np.zeros((B, N, D))
    for b in range(B):
        at = [(int(block_table[b][j // page_size]), j % page_size)
              for j in visible_tokens(kv_len[b], n_pinned, window, block_table.shape[1] * page_size)]
        at = [x for x in at if 0 <= x[0] < n_pages]
        if not at:
            continue
        page, off = np.array(at).T
        K, V = (np.asarray(x[page, off], dtype=np.float64) for x in (K_pages, V_pages))  # [tokens, N_kv, D]
        for h in range(N):
            g = h // (N // N_kv)
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (K[:, g] @ Q[b, h])
                if np.all(s == -np.inf):
                    continue
                w = np.exp(s - s.max())
                O[b, h] = (w[:, None] * V[:, g]).sum(0) / w.sum()
    return O
