"""CPU oracle for what surrounds attention in a step: tables, rotary rows, bounds of pages, their choice, attention over them.
TEST INFRASTRUCTURE ONLY, like ``paged_attention``: plain definitions in float64 (whole numbers as they are), no code shared with
the CUDA path.  Page images are in the logical layout [page][kv_head][slot][dim].

Pins (tests/test_step_oracle_pins.py): tables worked by hand and against a token-by-token walk; rotation keeps norms, composes
(positions a then b = position a + b) and depends on differences only under the inner product; a page's score is never below the
largest product with one of its keys; the choice by brute force over subsets; attention over all pages = paged_attention.attn_decode.
"""
from __future__ import annotations

import numpy as np

from .paged_attention import PagePool, attention_rows, widen

PAGE = 16


def step_tables(ctx, new, free, tables, total, num_pages, cursor=0):
    """Returns tables, cu, positions, slots, next lengths, next cursor, ok (False: something is recorded as out of bounds)."""
    tables = np.array(tables, dtype=np.int64).copy()
    width, ok = tables.shape[1], 0 <= cursor <= len(free)
    avail = len(free) - cursor if ok else 0
    cu, pos, slots, nxt = [0], np.zeros(total, np.int64), np.full(total, -1, np.int64), []
    taken = wanted = 0
    for i, (c, n) in enumerate(zip(ctx, new)):
        c, n = int(c), int(n)
        start = cu[-1]
        cu.append(start + max(n, 0))
        good = c >= 0 and n >= 0 and c + n <= width * PAGE and cu[-1] <= total
        need = -(-(c + n) // PAGE) - -(-c // PAGE) if good else 0
        wanted += need
        if need > 0 and wanted > avail:
            good = False
        nxt.append(c + n if good else c)
        if not good:
            ok = False
            continue
        first = taken
        if need > 0:
            taken = wanted
        for t in range(n):
            p = c + t
            b, owned = p // PAGE, -(-c // PAGE)
            pos[start + t] = p
            page = int(free[cursor + first + b - owned]) if b >= owned else int(tables[i, b])
            if not 0 <= page < num_pages:
                ok = False
                continue
            if b >= owned:
                tables[i, b] = page
            slots[start + t] = page * PAGE + p % PAGE
    return tables, np.minimum(cu, total), pos, slots, nxt, cursor + taken, ok


def rotate(x, positions, inv_freq, freq_axis=None, neighbours=False):
    """x [tokens][heads][D] float64; positions [axes][tokens]; returns the rotated rows, unrounded."""
    half = len(inv_freq)
    axis = np.zeros(half, np.int64) if freq_axis is None else np.asarray(freq_axis)
    theta = np.asarray(positions)[axis].T.astype(np.float64) * np.asarray(inv_freq, np.float64)[None, :]
    cos, sin = np.cos(theta)[:, None, :], np.sin(theta)[:, None, :]
    j = np.arange(half)
    a, b = (2 * j, 2 * j + 1) if neighbours else (j, j + half)
    y = np.array(x, dtype=np.float64)
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def page_bounds(pool: PagePool, slots, bounds):
    """bounds [pages][heads][2][D] float64, renewed for the pages of the slots."""
    bounds = bounds.copy()
    last = {}
    for s in slots:
        if s >= 0:
            last[int(s) // PAGE] = max(last.get(int(s) // PAGE, 0), int(s) % PAGE)
    for page, at in last.items():
        k = widen(pool.k[page, :, :at + 1])                                  # [heads][tokens][D]
        bounds[page, :, 0], bounds[page, :, 1] = np.min(k, axis=1), np.max(k, axis=1)   # (not a number: in both)
    return bounds


def page_scores(q, bounds):
    """q [G][D], bounds [pages][2][D], float64: the largest over the query rows of the sum of the larger side of every dim."""
    with np.errstate(invalid="ignore", over="ignore"):
        side = np.where(q[:, None, :] >= 0, q[:, None, :] * bounds[None, :, 1], q[:, None, :] * bounds[None, :, 0])
        return np.max(np.sum(side, axis=2), axis=0)


def select_pages(q_bits, bounds, tables, ctx, n_kv, n_select, n_first, n_last):
    """Lists [batch][heads][n_select] (-1 behind the count) and counts."""
    B, hq, D = q_bits.shape
    G = hq // n_kv
    q = widen(q_bits)
    out, counts = np.full((B, n_kv, n_select), -1, np.int64), np.zeros((B, n_kv), np.int64)
    for i in range(B):
        nb = max(0, -(-int(ctx[i]) // PAGE))
        for h in range(n_kv):
            forced = [b for b in range(nb) if b < n_first or b >= nb - n_last]
            others = list(range(n_first, nb - n_last))
            if nb <= n_select:
                chosen = list(range(nb))
            else:
                s = page_scores(q[i, h * G:(h + 1) * G], bounds[np.asarray(tables[i][:nb])[others], h])
                rank = [(0, 0.0, b) if np.isnan(v) else (1, -v, b) for v, b in zip(s, others)]
                chosen = sorted(forced + [r[2] for r in sorted(rank)[:n_select - len(forced)]])
            out[i, h, :len(chosen)] = chosen
            counts[i, h] = len(chosen)
    return out, counts


def decode_selected(pool: PagePool, q_bits, n_q_heads, tables, ctx, lists, counts, scale):
    B, _, D = q_bits.shape
    G = n_q_heads // pool.n_kv_heads
    q = widen(q_bits)
    out, lse = np.zeros((B, n_q_heads, D)), np.full((B, n_q_heads), -np.inf)
    for i in range(B):
        L = int(ctx[i])
        for h in range(pool.n_kv_heads):
            ks, vs = [], []
            for b in lists[i][h][:counts[i][h]]:
                if L <= 0 or not 0 <= b < -(-L // PAGE):
                    continue
                n, page = min(PAGE, L - int(b) * PAGE), int(tables[i][b])
                ks.append(widen(pool.k[page, h, :n]))
                vs.append(widen(pool.v[page, h, :n]))
            if not ks:
                continue
            k, v = np.concatenate(ks), np.concatenate(vs)
            rows = slice(h * G, (h + 1) * G)
            out[i, rows], lse[i, rows] = attention_rows(q[i, rows], k, v, np.full(G, len(k)), scale)
    return out, lse
