"""Oracle: paged key/value cache - plan of pages and slots, store, attention.

Test infrastructure only (see the package docstring).  Float64 and Python integers.

The paper does not specify attention or its cache (Sec. IV-A only overlaps transfers with it);
the operators serve requests of different lengths from one pool of pages:

* ``plan``   one request after the other: ended requests push their pages onto a stack, the
             others pop what they lack, until the first that does not fit;
* ``store``  a row per token and head into its slot: bf16, or E4M3 codes with a scale per row
             (``fp8``'s rule for a row of weights);
* ``attend`` softmax(scale q.K) V over the positions a token sees: up to its own, the last
             ``window`` (0: all) and the first ``sinks``, without pages whose id is out of range.
"""
from __future__ import annotations

import numpy as np

from . import fp8
from .attention import round_bf16

SERVED, ENDED, WAITS, INVALID = 0, 1, 2, 3


def _blocks(n, page):
    return -(-n // page)


def plan(cached, n_new, page, n_pages, table, T, free_pages, free_count):
    """Sequential replay.  table [R, max_blocks]; free_pages [n_pages].  Returns a dict of the
    outputs; the inputs stay as they are."""
    R, width = len(cached), table.shape[1]
    table, stack = table.copy(), [int(x) for x in free_pages]
    top = min(max(int(free_count), 0), n_pages)
    status = [SERVED] * R
    for r in range(R):
        c, n = int(cached[r]), int(n_new[r])
        if c < 0 or n < -1 or c + max(n, 0) > width * page:
            status[r] = INVALID
        elif n == -1:
            status[r] = ENDED
            for b in range(_blocks(c, page)):
                if top < n_pages:
                    stack[top] = int(table[r, b])
                    top += 1
    pushed = list(stack)
    got, tokens, waiting = [0] * R, 0, False
    for r in range(R):
        c, n = int(cached[r]), int(n_new[r])
        if status[r] != SERVED or n == 0:
            continue
        need = _blocks(c + n, page) - _blocks(c, page)
        if waiting or need > top or tokens + n > T:
            waiting, status[r] = True, WAITS
            continue
        for b in range(_blocks(c, page), _blocks(c + n, page)):
            top -= 1
            table[r, b] = stack[top]
        got[r] = n
        tokens += n
    cu = np.concatenate([[0], np.cumsum(got)]).astype(np.int64)
    slots, positions = np.full(T, -1, np.int64), np.full(T, -1, np.int64)
    t = 0
    for r in range(R):
        for i in range(got[r]):
            p = int(cached[r]) + i
            pid = int(table[r, p // page])
            positions[t] = p
            if 0 <= pid < n_pages:
                slots[t] = pid * page + p % page
            t += 1
    seq = [0 if status[r] == ENDED else min(max(int(cached[r]), 0), width * page) + got[r] for r in range(R)]
    return dict(block_table=table, free_pages=np.array(pushed, np.int64), free_count=top, cu_new=cu,
                seq_len=np.array(seq, np.int64), slot_map=slots, positions=positions,
                status=np.array(status, np.int64))


def quantise_row(x):
    """(codes, scale) of one row in float64: fp8's rule; NaN scale where a value is not finite."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), np.float32("nan")
    s = np.float32(np.abs(x).max() / fp8.MAX_FINITE)
    if s == 0:
        return np.zeros(len(x), np.uint8), s
    return fp8.encode(x / np.float64(s)), s


def store(rows, slot_map, page, pages, scales):
    """rows [T, G, hd] float64 into pages [n_pages, G, page, hd] (bf16 values as float64, or codes
    where scales [n_pages, G, page] is given), in place."""
    n_slots = pages.shape[0] * page
    for t, slot in enumerate(slot_map):
        if not 0 <= slot < n_slots:
            continue
        for g in range(rows.shape[1]):
            if scales is None:
                pages[slot // page, g, slot % page] = round_bf16(rows[t, g])
            else:
                c, s = quantise_row(rows[t, g])
                pages[slot // page, g, slot % page] = c
                scales[slot // page, g, slot % page] = s


def visible_positions(p, window, sinks):
    """Positions a query at position p sees, ascending."""
    j = np.arange(p + 1)
    return j if window == 0 else j[(j > p - window) | (j < sinks)]


def attend(q, k_pages, v_pages, cu_new, seq_len, table, window, sinks, scale, out):
    """q [T, H, hd]; pages [n_pages, G, page, hd] as float64 values.  Returns (out, size, peak): out
    [T, H, hd] with rows outside of the requests as given, 0 where all scores are -inf; size = sum of weight * |value| of every
    output; peak [T, H] = the largest sum of |scale q k| of a visible position."""
    n_pages, G, page, hd = k_pages.shape
    H = q.shape[1]
    out = np.array(out, np.float64)
    size, peak = np.zeros_like(out), np.zeros(out.shape[:2])
    for r in range(len(seq_len)):
        n = int(cu_new[r + 1] - cu_new[r])
        for i in range(n):
            t, p = int(cu_new[r]) + i, int(seq_len[r]) - n + i
            j = visible_positions(p, window, sinks)
            pid = np.asarray(table[r])[j // page].astype(np.int64)
            good = (pid >= 0) & (pid < n_pages)
            j, pid = j[good], pid[good]
            if len(j) == 0:
                out[t] = 0.0
                continue
            for g in range(G):
                K, V = k_pages[pid, g, j % page], v_pages[pid, g, j % page]
                for h in range(g * (H // G), (g + 1) * (H // G)):
                    s = (K @ q[t, h]) * scale
                    if s.max() == -np.inf:
                        out[t, h] = 0.0
                        continue
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[t, h] = w @ V
                    size[t, h] = w @ np.abs(V)
                    peak[t, h] = ((np.abs(K) @ np.abs(q[t, h])) * scale).max()
    return out, size, peak
