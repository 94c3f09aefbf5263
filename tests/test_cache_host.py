"""Checks that need no GPU of the operators around a paged cache: the oracle against other ways of writing the definitions down, the host
forms of the page bookkeeping against the oracle, long lives of a pool, refusals before any CUDA call, workspace sizes."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from oracle import loma_oracle as O
from paper_2401_09486_b200 import binding as L
from paper_2401_09486_b200 import build

INVALID, UNSUPPORTED, ALIGNMENT, CAPACITY, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return L.lib()


def i32(x, device="cpu"):
    return torch.tensor(np.asarray(x, dtype=np.int64), dtype=torch.int32, device=device)


# ------------------------------------------------------------------------------------------------ the 4-bit format
def test_kv4_values_by_hand():
    x = np.zeros(64)
    x[:6] = [15.0, -15.0, 1.0, 2.0, -13.99, 14.0]                # h = 1
    x[32:35] = [7.5, -0.1, 0.99]                                  # h = 0.5
    y = C.kv4_values(x)
    assert y[:7].tolist() == [15, -15, 1, 3, -13, 15, 1] and y[32:36].tolist() == [7.5, -0.5, 0.5, 0.5]
    assert C.kv4_steps(x).tolist() == [1.0, 0.5]


def test_kv4_values_properties():
    rng = np.random.default_rng(0)
    for dtype in (np.float64, np.float32):
        x = (rng.standard_normal((50, 128)) * 10.0 ** rng.integers(-30, 30, (50, 1))).astype(dtype).astype(np.float32).astype(np.float64)
        y, h = C.kv4_values(x), np.repeat(C.kv4_steps(x), 32, -1)
        assert (np.abs(x - y) <= h * (1 + 1e-12)).all() and (np.sign(y) * np.where(x == 0, 1, np.sign(x)) > 0).all()
        n = np.abs(y / h)
        assert (n == np.round(n)).all() and (n % 2 == 1).all() and n.max() == 15
        assert np.array_equal(C.kv4_values(y), y)                 # the outermost value is 15 h, so the steps come out again
    x = np.zeros(96)
    x[0], x[40] = np.nan, -np.inf
    assert np.isnan(C.kv4_values(x)[:64]).all() and (C.kv4_values(x)[64:] == 0).all()
    tiny = np.full(32, 2.0**-130)
    assert (C.kv4_values(tiny) == 0).all()
    big = np.full(32, 3e38)
    assert np.allclose(C.kv4_values(big), 3e38, rtol=2.0**-8)


def test_bf16_rounding_against_torch():
    x = torch.randn(10000, generator=torch.Generator().manual_seed(0)) * 10.0 ** torch.randint(-35, 35, (10000,), generator=torch.Generator().manual_seed(1))
    assert np.array_equal(C.bf16(x.numpy()), x.to(torch.bfloat16).double().numpy())


def test_decode_oracle_against_the_plain_decode():
    """Heads that are not grouped, all entries in the tail: the pinned decode step."""
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 2, 4, 1, 64))
    kc, vc = rng.standard_normal((2, 2, 4, 9, 64))
    want, lse, wk, wv = O.decode_attn(q, k, v, kc, vc, 6)
    none = [np.zeros((4, 0, 64))] * 2
    o, l2, _ = C.decode_attn_kv4(q[:, :, 0], none, none, list(wk[:, :, :7]), list(wv[:, :, :7]))
    assert np.allclose(o, want[:, :, 0]) and np.allclose(l2, np.asarray(lse).reshape(l2.shape))
    # ... and split between memory and tail
    o3, l3, _ = C.decode_attn_kv4(q[:, :, 0], list(wk[:, :, :5]), list(wv[:, :, :5]), list(wk[:, :, 5:7]), list(wv[:, :, 5:7]))
    assert np.allclose(o3, o) and np.allclose(l3, l2)


# ------------------------------------------------------------------------------------------------ pages
def pool_case(seed, B, M, ps, n_pages, bad=0.0):
    """Random tables of a pool whose pages have one owner, or several where rows share their beginnings."""
    rng = np.random.default_rng(seed)
    ids = rng.permutation(n_pages)
    lens = rng.integers(-1, M * ps + 2, B)
    held = np.minimum(-(-np.maximum(lens, 0) // ps) + rng.integers(0, 2, B), M)
    fixed = np.where(lens > 0, rng.integers(0, np.maximum(lens, 0) + 1), 0)
    table, at = np.full((B, M), -1), 0
    for b in range(B):
        first = 0
        if b and rng.random() < 0.5:
            a = int(rng.integers(0, b))
            first = int(min(held[a], held[b], fixed[a] // ps, fixed[b] // ps))
            table[b, :first] = table[a, :first]
        want = int(min(held[b] - first, max(0, n_pages - at)))
        table[b, first: first + want] = ids[at: at + want]
        at += want
        held[b] = first + want
    lens = np.minimum(lens, held * ps)
    lens = np.where((lens == 0) & (rng.random(B) < 0.3), -1, lens)
    fixed = np.minimum(fixed, np.maximum(lens, 0))
    refs = np.zeros(n_pages, dtype=np.int64)
    for b in range(B):
        for p in table[b, : held[b]]:
            refs[p] += 1
    refs = np.maximum(refs - 1, 0)
    if bad:
        table = np.where(rng.random(table.shape) < bad, rng.choice([-1, -(2**31), n_pages, 2**31 - 1], table.shape), table)
    free = np.concatenate([ids[:at], ids[at:]])          # the places in front of `at` are of pages handed out
    return lens, fixed, held, table, refs, free, at, rng


def run_release(case, keep, ps, device="cpu", in_place=False):
    lens, fixed, held, table, refs, free, taken, _ = case
    hd, tb, rf, fr, tk = i32(held, device), i32(table, device).reshape(len(held), -1), i32(refs, device), i32(free, device), i32([taken], device)
    out = hd if in_place else torch.full_like(hd, -77)
    counts = i32([-7] * 4, device)
    L.loma_paged_release(i32(keep, device), hd, tb, ps, out, rf, fr, tk, counts)
    return tb, out, rf, fr, tk, counts


def check_release(got, want):
    for g, w in zip(got, want):
        assert g.cpu().flatten().tolist() == np.asarray(w).reshape(-1).tolist()


def run_fork(case, parents, ps, max_copies, device="cpu", with_fixed=True, with_held=True):
    lens, fixed, held, table, refs, free, taken, _ = case
    B, M = table.shape
    rf, fr, tk = i32(refs, device), i32(free, device), i32([taken], device)
    new = lambda *s: torch.full(s, -77, dtype=torch.int32, device=device)  # noqa: E731
    out, lo, ho, src, dst, counts = new(B, M), new(B), new(B), new(max_copies), new(max_copies), new(4)
    ws = torch.full((max(1, L.loma_paged_fork_workspace_bytes(B)),), 171, dtype=torch.uint8, device=device)
    tb = i32(table, device).reshape(B, M)
    L.loma_paged_fork(i32(parents, device), i32(lens, device), i32(fixed, device) if with_fixed else None, i32(held, device) if with_held else None,
                      tb, ps, out, lo, ho, rf, fr, tk, src, dst, counts, workspace=ws)
    assert tb.flatten().tolist() == table.reshape(-1).tolist()
    return out, lo, ho, rf, fr, tk, (src, dst), counts


def check_fork(got, want):
    for i, (g, w) in enumerate(zip(got, want)):
        if i == 6:
            n = g[0].numel()
            pairs = list(zip(g[0].tolist(), g[1].tolist()))
            assert pairs[: len(w)] == [tuple(x) for x in w] and pairs[len(w):] == [(-1, -1)] * (n - len(w))
        else:
            assert g.cpu().flatten().tolist() == np.asarray(w).reshape(-1).tolist(), i


def run_compact(case, max_copies, device="cpu"):
    lens, fixed, held, table, refs, free, taken, _ = case
    tb, rf, fr, tk = i32(table, device).reshape(table.shape), i32(refs, device), i32(free, device), i32([taken], device)
    new = lambda n: torch.full((n,), -77, dtype=torch.int32, device=device)  # noqa: E731
    pm, src, dst, counts = new(len(refs)), new(max_copies), new(max_copies), new(4)
    L.loma_paged_compact(i32(held, device), tb, rf, fr, tk, pm, src, dst, counts)
    return tb, rf, fr, tk, pm, (src, dst), counts


def check_compact(got, want):
    check_fork((*got[:5], got[4], got[5], got[6]), (*want[:5], want[4], want[5], want[6]))


def parents_of(case, mode):
    rng, B = case[7], len(case[0])
    if mode == "any":
        return rng.integers(-1, B + 1, B)
    if mode == "one":
        return np.full(B, int(rng.integers(0, B)))
    return np.arange(B)


PAGE_CASES = [(1, 1, 1, 1), (1, 3, 4, 9), (6, 4, 4, 40), (5, 7, 16, 20), (37, 6, 8, 300), (64, 12, 16, 500), (9, 0, 4, 3), (3, 5, 2, 0)]


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("B,M,ps,n_pages", PAGE_CASES)
def test_host_pages_match_oracle(lib, B, M, ps, n_pages, seed):
    bad = 0.15 if seed >= 4 else 0.0
    case = pool_case(seed, B, M, ps, n_pages, bad)
    lens, fixed, held, table, refs, free, taken, rng = case
    keep = np.where(rng.random(B) < 0.3, -1, rng.integers(0, M * ps + 2, B))
    check_release(run_release(case, keep, ps, in_place=seed % 2 == 0), C.release(keep, held, table, ps, refs, free, taken))
    most = [0, 3, 500][seed % 3]
    for mode in ("any", "one", "same"):
        parents = parents_of(case, mode)
        f, h = (None if seed == 1 else fixed), (None if seed == 2 else held)
        check_fork(run_fork(case, parents, ps, most, with_fixed=f is not None, with_held=h is not None),
                   C.fork(parents, lens, f, h, table, ps, refs, free, taken, most))
    check_compact(run_compact(case, most), C.compact(held, table, refs, free, taken, most))


def test_fork_that_changes_nothing(lib):
    case = pool_case(3, 8, 5, 4, 60)
    out, lo, ho, rf, fr, tk, _, counts = run_fork(case, np.arange(8), 4, 10)
    held = case[2]
    assert [row[:h] for row, h in zip(out.tolist(), held)] == [row[:h] for row, h in zip(case[3].tolist(), held)]
    assert rf.tolist() == case[4].tolist() and int(tk) == case[6] and counts.tolist() == [0, 0, 0, 0] and ho.tolist() == held.tolist()


def test_lists_that_are_too_short(lib):
    """A list without room for what comes back, and one that cannot give what children need."""
    table, held = np.array([[0, 1, 2], [3, 4, -1]]), np.array([3, 2])
    case = (np.array([6, 4]), np.array([0, 0]), held, table, np.zeros(6, dtype=np.int64), np.array([5]), 0, None)
    check_release(run_release(case, [0, 0], 2), C.release([0, 0], held, table, 2, [0] * 6, [5], 0))
    got = run_release(case, [0, 0], 2)
    assert got[5].tolist() == [0, 5, 5, 0] and got[3].tolist() == [5] and int(got[4]) == 0
    out, _, ho, _, _, tk, (src, dst), counts = run_fork(case, [0, 0], 2, 8)       # row 1 ends, its pages have nowhere to go; one page for three
    assert out.tolist() == [[0, 1, 2], [5, -1, -1]] and ho.tolist() == [3, 1] and counts.tolist() == [1, 2, 2, 2] and int(tk) == 1
    assert src.tolist()[:2] == [0, -1] and dst.tolist()[:2] == [5, -1]


class Life:
    """A pool's life through the binding, with what every page holds kept beside it: sequence contents must survive."""

    def __init__(self, seed, B, M, ps, n_pages, device, copy):
        self.rng, self.B, self.M, self.ps, self.n, self.dev, self.copy = np.random.default_rng(seed), B, M, ps, n_pages, device, copy
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        self.table, self.held, self.refs = z(B, M) - 1, z(B), z(n_pages)
        self.free, self.taken = i32(self.rng.permutation(n_pages), device), z(1)
        self.lens = z(B) - 1
        self.want = [[] for _ in range(B)]       # entry by entry
        self.fixed = [0] * B
        self.pool = torch.full((n_pages, ps, 4), -1, dtype=torch.int32, device=device)   # an entry is 16 bytes, all alike
        self.next = 0

    def extend(self):
        room = self.M * self.ps
        new = [int(self.rng.integers(0, 2 * self.ps)) if n >= 0 and self.rng.random() < 0.7 else 0 for n in self.lens.tolist()]
        new = [min(m, room - max(n, 0)) for m, n in zip(new, self.lens.tolist())]
        rows = sum(new)
        e = lambda n: torch.empty(n, dtype=torch.int32, device=self.dev)  # noqa: E731
        slots, seq, pos, rs, pg = e(rows), e(rows), e(rows), e(self.B + 1), e(self.B + 1)
        L.loma_paged_extend(self.lens, i32(new, self.dev), self.held, None, self.free, self.taken, self.table, self.ps, rs, pg, self.held, slots, seq, pos)
        if int(pg[-1]) > self.n:                  # out of pages: everybody who got too few is ended
            have = self.held.tolist()
            new = [m if -(-(max(n, 0) + m) // self.ps) <= h else None for m, n, h in zip(new, self.lens.tolist(), have)]
        vals, at = [], 0
        keep = []
        flat = []
        for b, m in enumerate(new):
            cnt = int(rs[b + 1]) - int(rs[b])
            if m is None:
                at += cnt
                keep.append(0)
                continue
            for i in range(m):
                flat.append((at + i, self.next))
                self.want[b].append(self.next)
                self.next += 1
            at += cnt
            keep.append(-1)
        if flat:
            idx = torch.tensor([x for x, _ in flat], device=self.dev)
            vals = i32([y for _, y in flat], self.dev)
            s = slots[idx].long()
            assert (s >= 0).all()
            self.pool.view(-1, 4)[s] = vals[:, None].expand(-1, 4)
        self.lens = i32([-1 if m is None else (n + m if n >= 0 else n) for m, n in zip(new, self.lens.tolist())], self.dev)
        if any(k == 0 for k in keep):
            for b, k in enumerate(keep):
                if k == 0:
                    self.want[b], self.fixed[b] = [], 0
            self.release(keep)

    def release(self, keep):
        counts = torch.empty(4, dtype=torch.int32, device=self.dev)
        L.loma_paged_release(i32(keep, self.dev), self.held, self.table, self.ps, self.held, self.refs, self.free, self.taken, counts)
        assert counts.tolist()[2] == 0

    def shrink(self):
        """Compress steps (entries from the fixed ones on are rewritten), and requests that end."""
        keep, lens = [], self.lens.tolist()
        for b in range(self.B):
            x = self.rng.random()
            if lens[b] < 0:
                keep.append(-1)
            elif x < 0.15:
                keep.append(0)
                lens[b], self.want[b], self.fixed[b] = -1, [], 0
            elif x < 0.5:
                n = self.fixed[b] + (lens[b] - self.fixed[b]) // 3
                for e in range(self.fixed[b], n):
                    page = int(self.table[b, e // self.ps])
                    self.pool[page, e % self.ps] = self.next
                    self.want[b][e] = self.next
                    self.next += 1
                lens[b], self.want[b], self.fixed[b] = n, self.want[b][:n], n
                keep.append(n)
            else:
                keep.append(-1)
        self.lens = i32(lens, self.dev)
        self.release(keep)

    def fork(self):
        lens = self.lens.tolist()
        live = [b for b in range(self.B) if lens[b] >= 0]
        parents = [int(self.rng.choice(live)) if live and self.rng.random() < 0.4 else (b if lens[b] >= 0 else -1) for b in range(self.B)]
        most = self.B * self.M
        e = lambda *s: torch.empty(s, dtype=torch.int32, device=self.dev)  # noqa: E731
        out, lo, ho, src, dst, counts = e(self.B, self.M), e(self.B), e(self.B), e(most), e(most), e(4)
        ws = torch.empty(L.loma_paged_fork_workspace_bytes(self.B), dtype=torch.uint8, device=self.dev)
        L.loma_paged_fork(i32(parents, self.dev), self.lens, i32(self.fixed, self.dev), self.held, self.table, self.ps, out, lo, ho, self.refs, self.free,
                          self.taken, src, dst, counts, workspace=ws)
        self.copy(self.pool, src, dst, counts)
        self.want = [list(self.want[p]) if p >= 0 else [] for p in parents]
        self.fixed = [self.fixed[p] if p >= 0 else 0 for p in parents]
        self.table, self.lens, self.held = out, lo, ho
        if counts.tolist()[3]:                    # whoever lacks pages ends
            keep = []
            for b in range(self.B):
                short = -(-max(int(lo[b]), 0) // self.ps) > int(ho[b])
                keep.append(0 if short else -1)
                if short:
                    self.want[b], self.fixed[b] = [], 0
            self.lens = i32([-1 if k == 0 else n for k, n in zip(keep, self.lens.tolist())], self.dev)
            self.release(keep)

    def compact(self):
        most = [3, self.n][int(self.rng.integers(0, 2))]
        e = lambda n: torch.empty(n, dtype=torch.int32, device=self.dev)  # noqa: E731
        pm, src, dst, counts = e(self.n), e(most), e(most), e(4)
        L.loma_paged_compact(self.held, self.table, self.refs, self.free, self.taken, pm, src, dst, counts)
        self.copy(self.pool, src, dst, counts)
        if counts.tolist()[3] == 0:
            named = [p for row, h in zip(self.table.tolist(), self.held.tolist()) for p in row[:h]]
            assert sorted(set(named)) == list(range(len(set(named))))

    def check(self):
        table, held, lens = self.table.tolist(), self.held.tolist(), self.lens.tolist()
        owners = [0] * self.n
        for b in range(self.B):
            for p in table[b][: held[b]]:
                owners[p] += 1
        free = self.free.tolist()[int(self.taken):]
        assert len(set(free)) == len(free) and all(owners[p] == 0 for p in free)
        assert len(free) + sum(o > 0 for o in owners) == self.n                    # no page is lost
        assert self.refs.tolist() == [max(o - 1, 0) for o in owners]
        pool = self.pool.cpu()
        for b in range(self.B):
            if lens[b] < 0:
                assert held[b] == 0
                continue
            assert len(self.want[b]) == lens[b]
            got = [pool[table[b][e // self.ps], e % self.ps].tolist() for e in range(lens[b])]
            assert got == [[x] * 4 for x in self.want[b]]

    def run(self, steps):
        self.lens = i32([0] * self.B, self.dev)
        for _ in range(steps):
            for act in self.rng.choice(["extend", "extend", "shrink", "fork", "compact", "start"], 3):
                if act == "start":
                    self.lens = i32([0 if n < 0 and self.rng.random() < 0.5 else n for n in self.lens.tolist()], self.dev)
                else:
                    getattr(self, act)()
            self.check()


def host_copy(pool, src, dst, counts):
    n = int(counts[0])
    s, d = src[:n].long(), dst[:n].long()
    assert not set(s.tolist()) & set(d.tolist()) and len(set(d.tolist())) == n
    pool[d] = pool[s].clone()


@pytest.mark.parametrize("seed,B,M,ps,n_pages", [(0, 6, 8, 4, 200), (1, 6, 8, 4, 30), (2, 12, 5, 16, 45), (3, 3, 20, 1, 40), (4, 16, 6, 8, 60)])
def test_a_pools_life_on_the_host(lib, seed, B, M, ps, n_pages):
    Life(seed, B, M, ps, n_pages, "cpu", host_copy).run(25)


# ------------------------------------------------------------------------------------------------ refusals (no CUDA call is made)
def z(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


def p(t):
    return ctypes.c_void_p(t.data_ptr())


def refuses(lib, name, good, changes):
    """`good`: the arguments of a call that would pass the checks; each change is (positions -> values, expected status)."""
    fn = getattr(lib, name)
    for change, status in changes:
        args = list(good)
        for i, v in change.items():
            args[i] = v
        assert fn(*args) == status, (name, change)


def test_release_refusals(lib):
    B, M, n = 3, 4, 8
    t = dict(keep=z(B), held=z(B), table=z(B, M), out=z(B), refs=z(n), free=z(n), taken=z(1), counts=z(4))
    good = [B, 4, M, n, n, p(t["keep"]), p(t["held"]), p(t["table"]), p(t["out"]), p(t["refs"]), p(t["free"]), p(t["taken"]), p(t["counts"]), 0, None]
    assert lib.loma_paged_release(*good) == 0
    odd = ctypes.c_void_p(t["held"].data_ptr() + 2)
    refuses(lib, "loma_paged_release", good, [({0: -1}, INVALID), ({1: 3}, INVALID), ({1: 0}, INVALID), ({1: 131072}, INVALID), ({2: -1}, INVALID), ({2: 2**30}, INVALID),
                                              ({3: -1}, INVALID), ({4: -1}, INVALID), *[({i: None}, INVALID) for i in range(5, 13)], ({6: odd}, ALIGNMENT),
                                              ({8: p(t["keep"])}, INVALID), ({9: p(t["free"])}, INVALID), ({11: p(t["counts"])}, INVALID),
                                              ({7: p(t["refs"])}, INVALID)])
    good[8] = good[6]
    assert lib.loma_paged_release(*good) == 0


def test_fork_refusals(lib):
    B, M, n, mc = 3, 4, 8, 5
    t = {k: z(*s) for k, s in dict(par=(B,), lens=(B,), fixed=(B,), held=(B,), table=(B, M), out=(B, M), lo=(B,), ho=(B,), refs=(n,), free=(n,), taken=(1,), src=(mc,),
                                   dst=(mc,), counts=(4,), ws=(2 * B,)).items()}
    good = [B, 4, M, n, n, mc] + [p(t[k]) for k in ("par", "lens", "fixed", "held", "table", "out", "lo", "ho", "refs", "free", "taken", "src", "dst", "counts", "ws")] \
        + [8 * B, 0, None]
    assert lib.loma_paged_fork(*good) == 0
    refuses(lib, "loma_paged_fork", good, [({0: -1}, INVALID), ({1: 12}, INVALID), ({5: -1}, INVALID), *[({i: None}, INVALID) for i in (6, 7, 10, 11, 12, 13, 14, 15, 16, 17, 18, 19)],
                                           ({11: good[10]}, INVALID), ({12: good[7]}, INVALID), ({13: good[9]}, INVALID), ({17: good[18]}, INVALID), ({20: None}, WORKSPACE),
                                           ({21: 8 * B - 1}, WORKSPACE), ({20: good[14]}, INVALID), ({8: ctypes.c_void_p(t["fixed"].data_ptr() + 1)}, ALIGNMENT)])
    for i in (8, 9):
        args = list(good)
        args[i] = None
        assert lib.loma_paged_fork(*args) == 0
    assert lib.loma_paged_fork_workspace_bytes(0) == 0 and lib.loma_paged_fork_workspace_bytes(-3) == 0


def test_compact_refusals(lib):
    B, M, n, mc = 3, 4, 8, 5
    t = {k: z(*s) for k, s in dict(held=(B,), table=(B, M), refs=(n,), free=(n,), taken=(1,), pm=(n,), src=(mc,), dst=(mc,), counts=(4,)).items()}
    good = [B, M, n, n, mc] + [p(t[k]) for k in ("held", "table", "refs", "free", "taken", "pm", "src", "dst", "counts")] + [0, None]
    assert lib.loma_paged_compact(*good) == 0
    refuses(lib, "loma_paged_compact", good, [({0: -1}, INVALID), ({2: -1}, INVALID), ({3: -2}, INVALID), ({4: -1}, INVALID), *[({i: None}, INVALID) for i in range(5, 14)],
                                              ({10: good[7]}, INVALID), ({11: good[12]}, INVALID), ({6: ctypes.c_void_p(t["table"].data_ptr() + 2)}, ALIGNMENT)])


def test_copy_refusals(lib):
    pool, src = torch.zeros(4, 64, dtype=torch.uint8), z(3)
    pools, sizes = (ctypes.c_void_p * 2)(pool.data_ptr(), pool.data_ptr()), (ctypes.c_int64 * 2)(64, 64)
    good = [2, pools, sizes, 4, p(src), p(src), p(src), 3, None]
    bad_pool, bad_size = (ctypes.c_void_p * 2)(pool.data_ptr(), pool.data_ptr() + 8), (ctypes.c_int64 * 2)(64, 24)
    refuses(lib, "loma_paged_copy", good, [({0: -1}, INVALID), ({3: -1}, INVALID), ({7: -1}, INVALID), ({1: None}, INVALID), ({2: None}, INVALID), ({4: None}, INVALID),
                                           ({5: None}, INVALID), ({6: None}, INVALID), ({1: (ctypes.c_void_p * 2)(pool.data_ptr(), None)}, INVALID), ({1: bad_pool}, ALIGNMENT),
                                           ({2: bad_size}, ALIGNMENT), ({2: (ctypes.c_int64 * 2)(64, -16)}, INVALID), ({2: (ctypes.c_int64 * 2)(64, 2**62)}, INVALID),
                                           ({4: p(pool)}, INVALID), ({6: ctypes.c_void_p(pool.data_ptr() + 16)}, INVALID), ({5: ctypes.c_void_p(src.data_ptr() + 1)}, ALIGNMENT)])
    for i in (0, 3, 7):
        args = list(good)
        args[i] = 0
        assert lib.loma_paged_copy(*args) == 0


def test_kv4_append_and_load_refusals(lib):
    B, H, D, l, ps, M, n = 2, 3, 128, 5, 16, 4, 6
    k, v = torch.zeros(B, H, l, D), torch.zeros(B, H, l, D)
    pool, table, lens = torch.zeros(n, L.loma_kv4_page_bytes(H, D, ps), dtype=torch.uint8), z(B, M), z(B)
    st = lambda *x: (ctypes.c_int64 * 3)(*x)  # noqa: E731
    s = st(H * l * D, l * D, D)
    good = [p(k), p(v), p(pool), p(table), p(lens), None, B, H, D, l, ps, M, n, s, s, 0, None]
    refuses(lib, "loma_kv4_append", good, [({6: -1}, INVALID), ({7: -1}, INVALID), ({8: 96}, UNSUPPORTED), ({9: -1}, INVALID), ({10: 8}, INVALID), ({10: 24}, INVALID),
                                           ({10: 131072}, INVALID), ({11: 2**28}, INVALID), ({12: 0}, INVALID), ({12: -1}, INVALID), *[({i: None}, INVALID) for i in (0, 1, 2, 3, 4, 13, 14)],
                                           ({13: st(H * l * D, l * D, D - 2)}, INVALID), ({13: st(0, l * D, D)}, INVALID), ({14: st(-1, l * D, D)}, INVALID),
                                           ({13: st(H * l * D, l * D + 2 * D, D + 2)}, INVALID), ({13: st(8 * l * D, l * D + 10, D + 2)}, ALIGNMENT), ({15: 7}, UNSUPPORTED),
                                           ({0: ctypes.c_void_p(k.data_ptr() + 4)}, ALIGNMENT), ({2: ctypes.c_void_p(pool.data_ptr() + 8)}, ALIGNMENT), ({0: p(pool)}, INVALID),
                                           ({5: ctypes.c_void_p(lens.data_ptr() + 2)}, ALIGNMENT)])
    for i in (6, 7, 9):
        args = list(good)
        args[i] = 0
        assert lib.loma_kv4_append(*args) == 0
    good = [p(pool), p(table), p(lens), p(k), p(v), B, H, D, l, ps, M, n, 0, None]
    refuses(lib, "loma_kv4_load", good, [({5: -1}, INVALID), ({7: 32}, UNSUPPORTED), ({8: -1}, INVALID), ({9: 4}, INVALID), ({11: 0}, INVALID), *[({i: None}, INVALID) for i in range(5)],
                                         ({3: p(v)}, INVALID), ({3: p(pool)}, INVALID), ({4: ctypes.c_void_p(v.data_ptr() + 8)}, ALIGNMENT), ({12: 2}, UNSUPPORTED)])
    args = list(good)
    args[8] = 0
    assert lib.loma_kv4_load(*args) == 0


def test_kv4_decode_refusals(lib):
    B, Hq, H, D, cap, ps, M, n = 2, 6, 3, 64, 9, 16, 4, 6
    q, o, kn, vn = torch.zeros(B, Hq, D), torch.zeros(B, Hq, D), torch.zeros(B, H, D), torch.zeros(B, H, D)
    kt, vt, lse = torch.zeros(B, H, cap, D), torch.zeros(B, H, cap, D), torch.zeros(B, Hq)
    pool, table, lens, tails = torch.zeros(n, L.loma_kv4_page_bytes(H, D, ps), dtype=torch.uint8), z(B, M), z(B), z(B)
    need = L.loma_decode_kv4_workspace_bytes(B, Hq, H, D, 60, 8)
    ws = torch.zeros(need, dtype=torch.uint8)
    good = [p(q), p(kn), p(vn), p(kt), p(vt), p(pool), p(table), p(o), p(lse), B, Hq, H, D, cap, p(tails), 8, ps, M, n, p(lens), 60, 0, 0.0, 0, p(ws), need, None]
    refuses(lib, "loma_decode_attn_kv4", good, [({9: -1}, INVALID), ({10: 7}, INVALID), ({11: 0}, INVALID), ({12: 80}, UNSUPPORTED), ({13: -1}, INVALID), ({15: 9}, CAPACITY),
                                                ({20: 65}, CAPACITY), ({15: -1}, INVALID), ({20: -1}, INVALID), ({16: 8}, INVALID), ({18: 0}, INVALID), ({21: 3}, UNSUPPORTED),
                                                *[({i: None}, INVALID) for i in (0, 1, 2, 3, 4, 5, 6, 7, 14, 19)], ({24: None}, WORKSPACE), ({25: need - 1}, WORKSPACE),
                                                ({0: ctypes.c_void_p(q.data_ptr() + 4)}, ALIGNMENT), ({14: ctypes.c_void_p(tails.data_ptr() + 1)}, ALIGNMENT),
                                                ({7: p(q)}, INVALID), ({3: p(vt)}, INVALID), ({8: p(o)}, INVALID), ({10: 2**24, 9: 2**10}, INVALID)])
    for i in (9, 10):
        args = list(good)
        args[i] = 0
        assert lib.loma_decode_attn_kv4(*args) == 0


def test_sizes(lib):
    assert L.loma_kv4_page_bytes(1, 128, 16) == 16 * 2 * 72 and L.loma_kv4_page_bytes(3, 64, 64) == 3 * 64 * 2 * 36
    assert [L.loma_kv4_page_bytes(*x) for x in ((0, 128, 16), (1, 96, 16), (1, 64, 8), (1, 64, 24))] == [0] * 4
    rng = np.random.default_rng(0)
    for _ in range(300):                          # a workspace made for the largest sizes does for the smaller ones
        H, g, D = int(rng.integers(1, 9)), int(rng.integers(1, 20)), int(rng.choice([64, 128]))
        B, mem, tail = int(rng.integers(1, 300)), int(rng.integers(0, 40000)), int(rng.integers(0, 500))
        big = L.loma_decode_kv4_workspace_bytes(B, H * g, H, D, mem, tail)
        for _ in range(5):
            small = L.loma_decode_kv4_workspace_bytes(int(rng.integers(1, B + 1)), H * g, H, D, int(rng.integers(0, mem + 1)), int(rng.integers(0, tail + 1)))
            assert 0 < small <= big


def test_binding_checks_shapes_and_types(lib):
    free, ref = z(4), z(4)
    args = lambda: [z(2), z(2), z(2, 3), 4, z(2), ref, free, z(1), z(4)]  # noqa: E731
    L.loma_paged_release(*args())
    for i, bad in ((0, z(3)), (1, z(2).long()), (2, z(3, 3)), (4, z(2).float()), (7, z(2)), (8, z(3)), (2, z(2, 6)[:, ::2])):
        a = args()
        a[i] = bad
        with pytest.raises(ValueError):
            L.loma_paged_release(*a)
    a = args()
    a[3] = 3
    with pytest.raises(L.LomaError):
        L.loma_paged_release(*a)
    k = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError):               # host tensors
        L.loma_kv4_append(k, k, torch.zeros(2, L.loma_kv4_page_bytes(2, 64, 16), dtype=torch.uint8), z(1, 2), 16, z(1))
    with pytest.raises(ValueError):
        L.loma_paged_copy([torch.zeros(4, 16)], z(2), z(2), z(1))


def test_sizes_beyond_64_bit_offsets_are_refused(lib):
    """Numbers that each pass their own bound but whose product does not fit; nothing is read."""
    big = 2**31 - 5000
    x, lens = torch.zeros(64), z(4)
    a, w = p(x), p(lens)
    wide = (ctypes.c_int64 * 3)(2**60, 2**29, 128)
    for B, H, l, n, st in ((big, big, 4, 6, wide), (1, big, 4, big, wide), (2, 1, 4, 6, (ctypes.c_int64 * 3)(2**60, 2**60, 128))):
        assert lib.loma_kv4_append(a, a, a, w, w, None, B, H, 128, l, 65536, 4, n, st, st, 0, None) == INVALID
    assert lib.loma_kv4_append(a, a, a, w, w, None, big, 1, 128, 4, 16, 2**27 - 1, 6, wide, wide, 0, None) == INVALID
    assert lib.loma_kv4_load(a, w, w, a, a, big, 1, 128, big, 16, 4, 6, 0, None) == INVALID
    assert lib.loma_kv4_load(a, w, w, a, a, 1, big, 128, 16, 65536, 4, big, 0, None) == INVALID
    assert lib.loma_decode_attn_kv4(a, a, a, a, a, a, w, a, None, 1, 2**20, 2**20, 128, big, w, 8, 65536, 4, big, w, 60, 0, 0.0, 0, a, 2**40, None) == INVALID
    for on_device in (0, 1):
        assert lib.loma_paged_release(big, 1, big, 6, 6, w, w, w, w, w, w, w, w, on_device, None) == INVALID
        assert lib.loma_paged_fork(big, 1, big, 6, 6, 4, *[w] * 15, 2**40, on_device, None) == INVALID
        assert lib.loma_paged_compact(big, big, 6, 6, 4, *[w] * 9, on_device, None) == INVALID


@pytest.mark.parametrize("scale,status", [(2.0**51, INVALID), (float("inf"), INVALID), (2.0**-51, INVALID), (1e-45, INVALID)])
def test_kv4_decode_refuses_scales_its_sums_cannot_carry(lib, scale, status):
    B, Hq, H, D, cap = 2, 6, 3, 64, 9
    q, kt, vt, o, lens, ws = torch.zeros(B, Hq, D), torch.zeros(B, H, cap, D), torch.zeros(B, H, cap, D), torch.zeros(B, Hq, D), z(B), torch.zeros(2**20, dtype=torch.uint8)
    for flags in (0, L.LOMA_FLAG_FORCE_GENERIC):
        for dtype in (0, 1):
            assert lib.loma_decode_attn_kv4(p(q), None, None, p(kt), p(vt), None, None, p(o), None, B, Hq, H, D, cap, p(lens), 8, 16, 0, 0, p(z(B)), 0, dtype, scale, flags, p(ws),
                                            2**20, None) == status


def apart_from_each_other(n):
    """Addresses of arrays that are not there: for calls that end on the host."""
    return [ctypes.c_void_p((i + 1) << 42) for i in range(n)]


@pytest.mark.skipif(torch.cuda.is_available(), reason="where the checks let a call through, the missing device has to end it")
def test_rows_and_columns_that_32_bit_steps_would_leave_are_refused(lib):
    """Kernels go over rows and columns in steps of up to 9472 in 32 bits: the last step must not pass INT_MAX."""
    top = 2**31 - 1 - 65536
    for B, M, refused in ((top + 1, 1, True), (2**31 - 2, 1, True), (2**31 - 9000, 0, True), (1, top + 1, True), (1, 2**31 - 1, True), (top, 1, False), (1, top, False), (0, top + 1, True)):
        for name, args in (("loma_paged_release", [B, 1, M, 6, 6, *apart_from_each_other(8), 1, None]),
                           ("loma_paged_fork", [B, 1, M, 6, 6, 4, *apart_from_each_other(15), 2**40, 1, None]),
                           ("loma_paged_compact", [B, M, 6, 6, 4, *apart_from_each_other(9), 1, None])):
            status = getattr(lib, name)(*args)
            assert (status == INVALID) == refused and status != 0, (name, B, M, status)


@pytest.mark.skipif(torch.cuda.is_available(), reason="where the checks let a call through, the missing device has to end it")
def test_kv4_decode_refuses_a_workspace_that_meets_its_tensors(lib):
    B, Hq, H, D, cap, ps, M, n = 2, 6, 3, 64, 9, 16, 4, 6
    need = L.loma_decode_kv4_workspace_bytes(B, Hq, H, D, 60, 8)
    names = dict(q=B * Hq * D * 4, kn=B * H * D * 4, vn=B * H * D * 4, kt=B * H * cap * D * 4, vt=B * H * cap * D * 4, pool=n * L.loma_kv4_page_bytes(H, D, ps), table=B * M * 4,
                 o=B * Hq * D * 4, lse=B * Hq * 4, tails=B * 4, mems=B * 4)
    at = dict(zip((*names, "ws"), (x.value for x in apart_from_each_other(12))))

    def status(ws, size=need, **without):
        a = {**{k: ctypes.c_void_p(v) for k, v in at.items()}, **without}
        return lib.loma_decode_attn_kv4(a["q"], a["kn"], a["vn"], a["kt"], a["vt"], a["pool"], a["table"], a["o"], a["lse"], B, Hq, H, D, cap, a["tails"], 8, ps, M, n, a["mems"], 60, 0,
                                        0.0, 0, ctypes.c_void_p(ws), size, None)

    assert status(at["ws"]) not in (0, INVALID, WORKSPACE)                      # the missing device
    for k, size in names.items():
        assert status(at[k]) == INVALID, k                                     # begins where the tensor does
        assert status(at[k] + size - 4 - (at[k] + size - 4) % 16) == INVALID, k   # ... in its last 16 bytes
        assert status(at[k] - need + 16) == INVALID, k                         # ends behind its beginning
        for ws in (at[k] - need // 16 * 16 - 16, at[k] + (size + 15) // 16 * 16):
            assert status(ws) not in (0, INVALID, WORKSPACE), k                # beside it
    assert status(at["lse"], lse=None) not in (0, INVALID, WORKSPACE)
    assert status(at["ws"], need - 1) == WORKSPACE


def test_release_refuses_one_array_for_keep_lens_and_the_counts(lib):
    """held_out may be held; keep_lens is an input of its own."""
    B, M, n = 3, 4, 8
    keep, held, table, refs, free, taken, counts = z(B), z(B) + 2, z(B, M), z(n), z(n), z(1), z(4)
    tail = [p(refs), p(free), p(taken), p(counts), 0, None]
    for keep_at, held_at, out_at, status in ((keep, held, held, 0), (held, held, held, INVALID), (keep, held, keep, INVALID), (held, held, keep, 0),
                                             (held, held, None, INVALID)):
        held.fill_(2)
        got = lib.loma_paged_release(B, 4, M, n, n, p(keep_at), p(held_at), p(table), p(out_at) if out_at is not None else ctypes.c_void_p(held.data_ptr() + 4), *tail)
        assert got == status
        if status:
            assert held.tolist() == [2] * B


def test_merge_reads_slots_of_workers_whatever_the_workspace_holds(lib, tmp_path):
    """A worker whose wait ran out notes nothing, and the merge behind it must stay in the workspace (tests/c_abi/kv4_parts_check.cu)."""
    exe = str(tmp_path / "kv4_parts_check")
    subprocess.run([build._nvcc(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.INCLUDE, "-I", build.CSRC,
                    os.path.join(build.ROOT, "tests", "c_abi", "kv4_parts_check.cu"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and "kv4 parts ok" in out.stdout, out.stdout + out.stderr
