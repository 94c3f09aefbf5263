"""What surrounds a paged cache, written out in fp64 NumPy and plain lists: memory entries held in 4 bits, decode attention over them
and an uncompressed tail, and the bookkeeping of pages (release, fork, compact).  Nothing here is shared with the CUDA library."""

from __future__ import annotations

import numpy as np

INT_MAX = 2**31 - 1
GROUP = 32


# ------------------------------------------------------------------------------------------------ 4 bits
def bf16(x):
    """fp32 values rounded to bf16 (to nearest, ties to even), as fp64; NaN and infinities stay."""
    f = np.asarray(x, dtype=np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(f), r, f).astype(np.float64)


def kv4_steps(x):
    """The steps of rows x [..., D], fp64 [..., D / 32]."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(all="ignore"):
        h = bf16(np.abs(g).max(-1).astype(np.float32) / np.float32(15))
    h = np.where(h < 2.0**-126, 0.0, h)
    return np.where(np.isfinite(g).all(-1) & np.isfinite(h), h, np.nan)


def kv4_values(x):
    """What rows x [..., D] stand for once they are held in 4 bits."""
    x = np.asarray(x, dtype=np.float64)
    h = kv4_steps(x)[..., None]
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(all="ignore"):
        m = sum((np.abs(g) >= 2 * h * k).astype(np.float64) for k in range(1, 8))
        y = np.where(g < 0, -1.0, 1.0) * (2 * m + 1) * h
    return y.reshape(x.shape)


# ------------------------------------------------------------------------------------------------ attention
def decode_attn_kv4(q, k_mem, v_mem, k_tail, v_tail, scale=None):
    """q [B, Hq, D]; k_mem, v_mem: per sequence [Hkv, n, D] (values); k_tail, v_tail: per sequence [Hkv, m, D], the new token last, or
    None for a slot without a request.  Returns o, lse and the weighted mean of |v| (NaN rows for idle slots)."""
    B, Hq, D = q.shape
    scale = D**-0.5 if scale is None else scale
    o, lse, o_abs = np.full((B, Hq, D), np.nan), np.full((B, Hq), np.nan), np.full((B, Hq, D), np.nan)
    for b in range(B):
        if k_tail[b] is None:
            continue
        k, v = np.concatenate([k_mem[b], k_tail[b]], 1), np.concatenate([v_mem[b], v_tail[b]], 1)
        g = Hq // k.shape[0]
        for hq in range(Hq):
            a = k[hq // g] @ q[b, hq] * scale
            top = a.max()
            with np.errstate(all="ignore"):
                e = np.exp(a - top)
                w = e / e.sum()
                o[b, hq] = w @ v[hq // g]
                o_abs[b, hq] = w @ np.abs(v[hq // g])
                lse[b, hq] = top + np.log(e.sum())
    return o, lse, o_abs


# ------------------------------------------------------------------------------------------------ pages
class Pool:
    """Free list, owners and tables as an allocator on the host keeps them.  refs: owners of a page beyond the first."""

    def __init__(self, refs, free_pages, taken):
        self.refs, self.free = [int(x) for x in refs], [int(x) for x in free_pages]
        self.taken = min(max(int(taken), 0), len(self.free))

    def real(self, page):
        return 0 <= page < len(self.refs)

    def settle(self):
        """Pages without an owner go to the front of the free list."""
        gone = [p for p, r in enumerate(self.refs) if r < 0]
        for p in gone:
            self.refs[p] = 0
        n = min(len(gone), self.taken)
        self.taken -= n
        self.free[self.taken: self.taken + n] = gone[:n]
        return len(gone), len(gone) - n


def clamp(x, lo, hi):
    return min(max(int(x), lo), hi)


def release(keep_lens, held, table, page_size, refs, free_pages, taken):
    """Returns (table, held_out, refs, free_pages, taken, counts)."""
    table = [[int(x) for x in r] for r in table]
    pool, M, held_out = Pool(refs, free_pages, taken), len(table[0]) if len(table) else 0, []
    for b, keep in enumerate(keep_lens):
        have = clamp(held[b], 0, M)
        stay = have if keep < 0 else min(have, -(-int(keep) // page_size))
        for j in range(stay, have):
            if pool.real(table[b][j]):
                pool.refs[table[b][j]] -= 1
            table[b][j] = -1
        held_out.append(stay)
    n, lost = pool.settle()
    return table, held_out, pool.refs, pool.free, pool.taken, [0, n, lost, 0]


def fork(parents, cache_lens, fixed_lens, held, table, page_size, refs, free_pages, taken, max_copies):
    """Returns (table_out, lens_out, held_out, refs, free_pages, taken, copies [(src, dst)], counts)."""
    table = [[int(x) for x in r] for r in table]
    B, M, ps = len(parents), len(table[0]) if len(table) else 0, page_size
    pool = Pool(refs, free_pages, taken)
    kids = {a: [b for b in range(B) if parents[b] == a] for a in range(B)}
    shape = []
    for a in range(B):
        n = clamp(cache_lens[a], 0, M * ps)
        f = n if fixed_lens is None else clamp(fixed_lens[a], 0, n)
        have = -(-n // ps) if held is None else clamp(held[a], 0, M)
        shape.append((have, min(f // ps, have), min(-(-n // ps), have)))
    for a in range(B):
        have, share, _ = shape[a]
        for j in range(share if kids[a] else have):
            if pool.real(table[a][j]):
                pool.refs[table[a][j]] += len(kids[a]) - 1
    n, lost = pool.settle()
    room, want, copies = min(len(pool.free) - pool.taken, max_copies), 0, []
    rows, lens_out, held_out = [], [], []
    for b in range(B):
        a = int(parents[b])
        if not 0 <= a < B:
            rows.append([-1] * M), lens_out.append(-1), held_out.append(0)
            continue
        have, share, used = shape[a]
        lens_out.append(int(cache_lens[a]))
        if b == (a if a in kids[a] else kids[a][0]):
            rows.append(table[a][:have] + [-1] * (M - have)), held_out.append(have)
            continue
        row, got = table[a][:share], 0
        for j in range(share, used):
            if want < room:
                page = pool.free[pool.taken + want]
                copies.append((table[a][j] if pool.real(table[a][j]) else -1, page))
                row.append(page)
                got += 1
            else:
                row.append(-1)
            want += 1
        rows.append(row + [-1] * (M - len(row))), held_out.append(share + got)
    return rows, lens_out, held_out, pool.refs, pool.free, pool.taken + len(copies), copies, [len(copies), n, lost, want - len(copies)]


def compact(held, table, refs, free_pages, taken, max_copies):
    """Returns (table, refs, free_pages, taken, page_map, copies, counts)."""
    table = [[int(x) for x in r] for r in table]
    pool, M = Pool(refs, free_pages, taken), len(table[0]) if len(table) else 0
    named = sorted({p for b, row in enumerate(table) for p in row[: clamp(held[b], 0, M)] if pool.real(p)})
    free = sorted({p for p in pool.free[pool.taken:] if pool.real(p)} - set(named))
    low = set(sorted(named + free)[: len(named)])
    src, dst = [p for p in named if p not in low], [p for p in free if p in low]
    moves = list(zip(src, dst))[:max_copies]
    page_map = list(range(len(pool.refs)))
    for s, d in moves:
        page_map[s] = d
        pool.refs[d], pool.refs[s] = pool.refs[s], 0
    rest = sorted((set(free) - {d for _, d in moves}) | {s for s, _ in moves})
    taken = len(pool.free) - len(rest)
    pool.free[taken:] = rest
    for b, row in enumerate(table):
        for j in range(clamp(held[b], 0, M)):
            if pool.real(row[j]):
                row[j] = page_map[row[j]]
    return table, pool.refs, pool.free, taken, page_map, moves, [len(moves), len(rest), len(named), len(src) - len(moves)]
