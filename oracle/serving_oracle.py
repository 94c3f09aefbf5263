"""Serving-step operators written out in fp64 NumPy: page tables and slot maps, the per-head RMS norm with the rotary
embedding and its gradients, and decode attention over a prefix that a batch shares.  Plain loops over sequences and
heads; nothing here is shared with the CUDA library."""

from __future__ import annotations

import numpy as np

from .loma_oracle import position_ids, rope_rotate

INT_MAX = 2**31 - 1


def paged_extend(cache_lens, new_lens, held, pos0, free_pages, taken, block_table, page_size, max_rows):
    """Returns (block_table, row_start, page_start, held_out, slots, row_seq, row_pos, taken) as an allocator that takes the
    sequences one after the other would leave them.  taken: pages of the list that are in use now, where the call was given such
    a count; without one the list's start is not kept and this is page_start[B]."""
    table = np.array(block_table, dtype=np.int64)
    B, M = table.shape
    ps = page_size
    row_start, page_start, held_out = [0], [0 if taken is None else min(max(int(taken), 0), INT_MAX)], []
    rows = []
    for b in range(B):
        n_have = min(max(int(cache_lens[b]), 0), M * ps)
        n_new = 1 if new_lens is None else max(int(new_lens[b]), 0)
        if cache_lens[b] < 0:
            n_new = 0
        h = -(-n_have // ps) if held is None else min(max(int(held[b]), 0), M)
        want = max(0, -(-min(n_have + n_new, M * ps) // ps) - h) if n_new > 0 else 0
        got = 0
        for i in range(want):
            at = page_start[-1] + i
            page = -1
            if at < len(free_pages):
                page = int(free_pages[at])
                got += 1
            table[b, h + i] = page
        for i in range(min(n_new, max(0, max_rows - row_start[-1]))):
            e = n_have + i
            slot = -1
            if e < M * ps and table[b, e // ps] >= 0 and table[b, e // ps] * ps + ps - 1 <= INT_MAX:
                slot = int(table[b, e // ps]) * ps + e % ps
            rows.append((slot, b, min((n_have if pos0 is None else int(pos0[b])) + i, INT_MAX)))
        row_start.append(min(row_start[-1] + n_new, INT_MAX))
        page_start.append(min(page_start[-1] + want, INT_MAX))
        held_out.append(h + got)
    rows += [(-1, -1, 0)] * (max_rows - len(rows))
    cols = [np.array([r[i] for r in rows], dtype=np.int64) for i in range(3)]
    after = page_start[-1] if taken is None else max(page_start[0], min(page_start[-1], len(free_pages)))
    return (table, np.array(row_start), np.array(page_start), np.array(held_out, dtype=np.int64), *cols, after)


def rms_norm(x, w=None, eps=1e-6):
    """x w / sqrt(mean of squares + eps) over the last axis."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if w is None else y * w


def norm_rope_rows(x, w, pos, eps=1e-6, base=10000.0):
    """Norm and rotation of rows x [..., S, D] at the ids pos [S]."""
    return rope_rotate(rms_norm(x, w, eps), pos, base)


def norm_rope_rows_bwd(x, w, pos, g, eps=1e-6, base=10000.0):
    """(dx, dw): the Jacobian of every row written as a matrix and applied to g, row by row."""
    D = x.shape[-1]
    w = np.ones(D) if w is None else w
    dx, dw = np.zeros(x.shape), np.zeros(D)   # contiguous, so that the reshape below is a view
    flat = [a.reshape(-1, x.shape[-2], D) for a in (x, g, dx)]
    eye = np.eye(D)
    for s in range(x.shape[-2]):
        R = rope_rotate(eye[None], np.full(D, pos[s]), base)[0]       # row d: the rotation of unit vector d
        for n in range(flat[0].shape[0]):
            row, u = flat[0][n, s], R @ flat[1][n, s]                 # u: gradient before the rotation
            r = 1.0 / np.sqrt(row @ row / D + eps)
            jac = r * eye - np.outer(row, row) * r**3 / D             # d(x r) / dx
            flat[2][n, s] = jac @ (w * u)
            dw += u * row * r
    return dx, dw


def qk_norm_rope(q, k, wq, wk, n_chunks, c, t, tail_read=0, flags=0, eps=1e-6, base=10000.0, position_type="intermittent"):
    pos = position_ids(n_chunks, c, t, tail_read, flags, position_type)
    return norm_rope_rows(q, wq, pos, eps, base), norm_rope_rows(k, wk, pos, eps, base)


def qk_norm_rope_bwd(q, k, wq, wk, gq, gk, n_chunks, c, t, tail_read=0, flags=0, eps=1e-6, base=10000.0,
                     position_type="intermittent"):
    """(dq, dk, dwq, dwk)"""
    pos = position_ids(n_chunks, c, t, tail_read, flags, position_type)
    dq, dwq = norm_rope_rows_bwd(q, wq, pos, gq, eps, base)
    dk, dwk = norm_rope_rows_bwd(k, wk, pos, gk, eps, base)
    return dq, dk, dwq, dwk


def qk_norm_rope_append(q, k, v, wq, wk, k_pool, v_pool, slots, positions, eps=1e-6, base=10000.0):
    """q [T, Hq, D], k, v [T, Hk, D]; returns (q_out, k_pool, v_pool)."""
    q_out = np.zeros_like(q)
    k_pool, v_pool = k_pool.copy(), v_pool.copy()
    n_pages, _, ps, _ = k_pool.shape
    for r in range(q.shape[0]):
        q_out[r] = norm_rope_rows(q[r][:, None], wq, [positions[r]], eps, base)[:, 0]
        if 0 <= slots[r] < n_pages * ps:
            k_pool[slots[r] // ps, :, slots[r] % ps] = norm_rope_rows(k[r][:, None], wk, [positions[r]], eps, base)[:, 0]
            v_pool[slots[r] // ps, :, slots[r] % ps] = v[r]
    return q_out, k_pool, v_pool


def decode_attn_shared(q, k_own, v_own, k_prefix, v_prefix, scale=None):
    """q [B, Hq, D]; k_own[b], v_own[b]: [Hkv, rows, D], the own entries and the new token of sequence b, or None (no
    request); k_prefix, v_prefix [Hkv, P, D].  Returns (o, lse, o_abs): o_abs is the same mean over |v|."""
    B, Hq, D = q.shape
    Hkv = k_prefix.shape[0]
    g = Hq // Hkv
    scale = D**-0.5 if scale is None else scale
    o, o_abs, lse = np.zeros_like(q), np.zeros_like(q), np.zeros((B, Hq))
    for b in range(B):
        if k_own[b] is None:
            continue
        for hq in range(Hq):
            keys = np.concatenate([k_prefix[hq // g], k_own[b][hq // g]])
            vals = np.concatenate([v_prefix[hq // g], v_own[b][hq // g]])
            a = keys @ q[b, hq] * scale
            top = a.max()
            e = np.exp(a - top)
            o[b, hq] = e @ vals / e.sum()
            o_abs[b, hq] = e @ np.abs(vals) / e.sum()
            lse[b, hq] = top + np.log(e.sum())
    return o, lse, o_abs
