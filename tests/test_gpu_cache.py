"""Parity of the operators around a paged cache with the oracle: page bookkeeping (exact), memory entries in 4 bits (exact), and decode
attention over them and the uncompressed tail.

Tolerances of the attention.  Memory entries are what they stand for, exactly.  A score is a dot product of D terms in fp32 times the scale,
off by at most (D + 8) 2^-23 of scale * sum |q_d k_d| (twice a half step per term: the tensor cores' sums are not rounded to nearest), so a weight is
off by that much of itself, and so is the weights' sum: twice.  Exponentials and the merge's factors take 2^-20 together, sums of n weights n 2^-23.  bf16 calls on the tensor
cores round each weight times its step to bf16 (half a step: 2^-8), and the output once (2^-8 of it); fp32 rounds the output by 2^-24."""

import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from oracle import loma_oracle as O
from paper_2401_09486_b200 import binding as L
from paper_2401_09486_b200 import build, synthetic
from tests import test_cache_host as H
from tests.test_cache_host import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GENERIC = L.LOMA_FLAG_FORCE_GENERIC
KINDS = [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, GENERIC)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build_library()
    L.lib()
    torch.cuda.set_device(0)
    yield
    assert L.loma_device_status() == 0


def npf(x):
    return x.detach().to("cpu").to(torch.float64).numpy()


def normal(shape, seed, dtype=torch.float32, std=1.0):
    return synthetic.normal_tensor(shape, seed, std, dtype).to(DEV)


def di32(x):
    return i32(x, DEV)


# ------------------------------------------------------------------------------------------------ pages
BIG = [(200, 20, 16, 3000), (1500, 8, 4, 9000), (3, 3000, 2, 5000), (20, 4, 16, 150000)]


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("B,M,ps,n_pages", H.PAGE_CASES + BIG)
def test_pages_match_oracle(B, M, ps, n_pages, seed):
    bad = 0.15 if seed >= 4 else 0.0
    case = H.pool_case(seed, B, M, ps, n_pages, bad)
    lens, fixed, held, table, refs, free, taken, rng = case
    keep = np.where(rng.random(B) < 0.3, -1, rng.integers(0, M * ps + 2, B))
    H.check_release(H.run_release(case, keep, ps, DEV, in_place=seed % 2 == 0), C.release(keep, held, table, ps, refs, free, taken))
    most = [0, 3, 20000][seed % 3]
    for mode in ("any", "one", "same"):
        parents = H.parents_of(case, mode)
        f, h = (None if seed == 1 else fixed), (None if seed == 2 else held)
        H.check_fork(H.run_fork(case, parents, ps, most, DEV, with_fixed=f is not None, with_held=h is not None),
                     C.fork(parents, lens, f, h, table, ps, refs, free, taken, most))
    H.check_compact(H.run_compact(case, most, DEV), C.compact(held, table, refs, free, taken, most))


@pytest.mark.parametrize("B,M", [(40, 30), (300, 20)])
def test_pages_of_a_pool_looked_at_in_stretches(B, M):
    """More pages than the words of a cluster's shared memory."""
    case = H.pool_case(7, B, M, 4, 1200000)
    lens, fixed, held, table, refs, free, taken, rng = case
    keep = np.where(rng.random(B) < 0.3, -1, rng.integers(0, M * 4 + 2, B))
    H.check_release(H.run_release(case, keep, 4, DEV), C.release(keep, held, table, 4, refs, free, taken))
    parents = H.parents_of(case, "any")
    H.check_fork(H.run_fork(case, parents, 4, 5000, DEV), C.fork(parents, lens, fixed, held, table, 4, refs, free, taken, 5000))
    for most in (100, 20000):
        H.check_compact(H.run_compact(case, most, DEV), C.compact(held, table, refs, free, taken, most))


@pytest.mark.parametrize("B,M,n_pages,room", [(600, 500, 300000, None), (200, 1400, 270001, None), (600, 500, 1200000, 1000), (600, 500, 300000, 0)])
def test_many_pages_released_at_once(B, M, n_pages, room):
    """So many that a launch over all SMs lists them; room: places in the list, fewer than pages that come back."""
    lens, fixed, held, table, refs, free, taken, rng = H.pool_case(B + M, B, M, 4, n_pages)
    if room is not None:
        taken = room
    case = (lens, fixed, held, table, refs, free, taken, rng)
    for keep in (np.where(rng.random(B) < 0.3, -1, rng.integers(0, M * 4 + 2, B)), np.zeros(B, dtype=np.int64), np.full(B, -1), np.where(np.arange(B) == 1, 0, -1)):
        H.check_release(H.run_release(case, keep, 4, DEV), C.release(keep, held, table, 4, refs, free, taken))


@pytest.mark.parametrize("taken", [-5, 0, 10**6])
def test_pages_of_an_empty_batch_and_a_start_out_of_range(taken):
    rf, fr, tk, ct = di32([0] * 5), di32([3, 1, 4]), di32([taken]), di32([-7] * 4)
    none, tab = di32([]), torch.empty(0, 3, dtype=torch.int32, device=DEV)
    L.loma_paged_release(none, none, tab, 4, none, rf, fr, tk, ct)
    at = min(max(taken, 0), 3)
    assert ct.tolist() == [0, 0, 0, 0] and int(tk) == at
    src, dst = di32([5, 5]), di32([5, 5])
    L.loma_paged_fork(none, none, None, None, tab, 4, tab.clone(), none.clone(), none.clone(), rf, fr, tk, src, dst, ct)
    assert ct.tolist() == [0, 0, 0, 0] and src.tolist() == [-1, -1]
    pm = torch.empty(5, dtype=torch.int32, device=DEV)
    L.loma_paged_compact(none, tab, rf, fr, tk, pm, src, dst, ct)
    want = C.compact([], [], [0] * 5, [3, 1, 4], at, 2)
    assert pm.tolist() == [0, 1, 2, 3, 4] and int(tk) == want[3] and fr.tolist()[want[3]:] == want[2][want[3]:] and ct.tolist() == want[6]


def test_pages_listed_twice_and_named_twice():
    """A page in the free list twice, one that is free and named, one that a row names twice: nothing is handed out twice."""
    held, table, refs, free = np.array([3, 2]), np.array([[6, 9, 6], [2, 7, -1]]), np.zeros(10, dtype=np.int64), np.array([5, 5, 2, 0, 8, 8])
    refs[6] = 1
    case = (np.array([12, 8]), np.array([0, 0]), held, table, refs, free, 0, None)
    H.check_compact(H.run_compact(case, 10, DEV), C.compact(held, table, refs, free, 0, 10))
    H.check_release(H.run_release(case, [0, 0], 4, DEV), C.release([0, 0], held, table, 4, refs, free, 0))


@pytest.mark.parametrize("seed,B,M,ps,n_pages", [(0, 6, 8, 4, 200), (1, 6, 8, 4, 30), (2, 12, 5, 16, 45), (4, 16, 6, 8, 60)])
def test_a_pools_life(seed, B, M, ps, n_pages):
    H.Life(seed, B, M, ps, n_pages, DEV, lambda pool, s, d, c: L.loma_paged_copy([pool], s, d, c[:1])).run(15)


@pytest.mark.parametrize("shapes", [[(9, 16)], [(9, 2, 16, 64), (9, 5, 16)], [(9, 4112)] * 3, [(9, 128, 1024)] * 2, [(9, 48)] * 70])
def test_copy(shapes):
    pools = [torch.randint(0, 256, s, dtype=torch.uint8, device=DEV) for s in shapes]
    for n, (src, dst) in ((5, ([0, 3, 3, 8, 5, 1], [1, 2, 4, 6, 5, 7])), (6, ([0, -1, 9, 3, 2, 1], [8, 2, 4, -1, 9, 2**31 - 1])), (0, ([0], [1])),
                          (-3, ([0], [1])), (99, ([4], [0]))):
        want = [x.clone() for x in pools]
        for w in want:
            for s, d in list(zip(src, dst))[: max(0, n)]:
                if 0 <= s < 9 and 0 <= d < 9:
                    w[d] = w[s]
        L.loma_paged_copy(pools, di32(src), di32(dst), di32([n]))
        assert all(torch.equal(x, w) for x, w in zip(pools, want))


def test_copy_offsets_beyond_32_bits():
    pool = torch.zeros(70, 2**26, dtype=torch.uint8, device=DEV)      # 4.7 GB
    pool[68] = torch.arange(2**26, device=DEV).to(torch.uint8)
    L.loma_paged_copy([pool], di32([68, 68]), di32([69, 1]), di32([2]))
    assert torch.equal(pool[69], pool[68]) and torch.equal(pool[1], pool[68]) and int(pool[67].max()) == 0


# ------------------------------------------------------------------------------------------------ 4 bits
def table_of(B, M, seed, extra=2):
    return di32(np.random.default_rng(seed).permutation(B * M + extra)[: B * M].reshape(B, M))


def new_pool(n_pages, Hkv, D, ps, fill=0):
    return torch.full((n_pages, L.loma_kv4_page_bytes(Hkv, D, ps)), fill, dtype=torch.uint8, device=DEV)


def stored(x, dtype):
    """What append and load make of x: the values of the format, rounded to the type."""
    return torch.from_numpy(C.kv4_values(npf(x))).to(dtype).to(torch.float64).numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,Hkv,D,ps,l,cap", [(1, 1, 64, 16, 1, 1), (1, 1, 128, 16, 1, 3), (3, 2, 128, 16, 37, 100), (5, 3, 64, 64, 130, 200), (2, 5, 128, 256, 16, 300),
                                              (9, 8, 64, 32, 5, 70), (40, 8, 128, 16, 16, 48)])
def test_append_and_load(B, Hkv, D, ps, l, cap, dtype):
    M = -(-cap // ps)
    rng = np.random.default_rng(B * 100 + l)
    lens = rng.integers(0, max(1, cap - l + 1), B)
    lens[::4] = np.where(np.arange(len(lens[::4])) % 2 == 1, -1, lens[::4])
    new = rng.integers(0, l + 1, B)
    new[0] = l
    pool, table = new_pool(B * M + 2, Hkv, D, ps, 255), table_of(B, M, B)           # bytes of 255: steps that are NaN
    before = pool.clone()
    base = [normal((B, l + 2, Hkv, D), 7 + i, dtype, 3.0) for i in (0, 1)]            # views: rows first, not contiguous
    k, v = (x.transpose(1, 2)[:, :, 1: l + 1] for x in base)
    L.loma_kv4_append(k, v, pool, table, ps, di32(lens), di32(new))
    kc, vc = (torch.full((B, Hkv, cap, D), 7.0, dtype=dtype, device=DEV) for _ in "kv")
    L.loma_kv4_load(pool, table, ps, di32(np.where(lens < 0, 0, lens + new)), kc, vc)
    for x, c in ((k, kc), (v, vc)):
        want, got = stored(x, dtype), npf(c)
        for b in range(B):
            n0 = lens[b]
            n1 = 0 if n0 < 0 else n0 + new[b]
            if n0 >= 0:
                assert np.array_equal(got[b, :, n0:n1], want[b, :, : new[b]])
            assert (got[b, :, max(n1, 0):] == 7.0).all()                              # rows behind the last
            if n0 > 0:
                assert np.isnan(got[b, :, :n0]).all()                                 # entries in front: as they were
    # nothing but the new rows has been written
    used = sum(int(new[b]) for b in range(B) if lens[b] >= 0) * Hkv * 2 * (D // 2 + D // 16)
    assert int((pool != before).sum()) <= used
    # new_lens left out
    again = before.clone()
    L.loma_kv4_append(k, v, again, table, ps, di32(lens))
    full = before.clone()
    L.loma_kv4_append(k, v, full, table, ps, di32(lens), di32(np.full(B, l + 5)))
    assert torch.equal(again, full)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_special_values(dtype):
    x = torch.randn(1, 2, 40, 128, generator=torch.Generator().manual_seed(0))
    x[0, 0, 0] = 0
    x[0, 0, 1, 5] = float("nan")
    x[0, 0, 2, 40] = float("inf")
    x[0, 0, 3, 127] = float("-inf")
    x[0, 0, 4] *= 1e-38
    x[0, 0, 5] *= 1e-40
    x[0, 0, 6] *= 3e37
    x[0, 0, 7] = 3.3e38
    x[0, 0, 8] = -0.0
    x[0, 0, 9] = 0.75
    x[0, 0, 10, :64] = torch.arange(64) - 32.0
    x[0, 0, 11, :32] = 2.0 * torch.arange(32) - 32                                    # values on the thresholds
    x[0, 0, 12, 3:] = 1e-30
    x = x.to(dtype).to(DEV)
    y = x.flip(1).contiguous()
    pool, table = new_pool(3, 2, 128, 64), di32([[1]])
    L.loma_kv4_append(x, y, pool, table, 64, di32([0]))
    kc, vc = torch.zeros_like(x), torch.zeros_like(x)
    L.loma_kv4_load(pool, table, 64, di32([40]), kc, vc)
    for a, c in ((x, kc), (y, vc)):
        assert np.array_equal(npf(c), stored(a, dtype), equal_nan=True)


def test_append_pages_out_of_range_and_past_the_table():
    B, Hkv, D, ps, M, n_pages = 4, 2, 64, 16, 2, 5
    k = normal((B, Hkv, 20, D), 1, torch.bfloat16)
    table = di32([[0, -1], [-5, 1], [n_pages, 2**31 - 1], [2, 3]])
    pool = new_pool(n_pages, Hkv, D, ps, 255)
    L.loma_kv4_append(k, k, pool, table, ps, di32([10, 10, 0, 25]))
    kc, vc = (torch.zeros(B, Hkv, 32, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    L.loma_kv4_load(pool, di32([[0, 4], [4, 1], [4, 4], [2, 3]]), ps, di32([32] * B), kc, vc)
    want, got = stored(k, torch.bfloat16), npf(kc)
    assert np.array_equal(got[0, :, 10:16], want[0, :, :6]) and np.isnan(got[0, :, 16:]).all()
    assert np.isnan(got[1, :, :16]).all() and np.array_equal(got[1, :, 16:30], want[1, :, 6:])
    assert np.isnan(got[2]).all() and np.isnan(npf(vc)[2]).all()
    assert np.array_equal(got[3, :, 25:32], want[3, :, :7]) and np.isnan(got[3, :, :25]).all()
    # reads clamp page numbers to the pool
    L.loma_kv4_load(pool, table, ps, di32([0, 32, 32, 0]), kc, vc)
    assert torch.equal(kc[2, :, :16].isnan(), torch.ones_like(kc[2, :, :16], dtype=torch.bool))


def test_kv4_offsets_beyond_32_bits():
    ps, D = 16, 128
    n = 2**32 // L.loma_kv4_page_bytes(1, D, ps) + 5
    pool = torch.zeros(n, L.loma_kv4_page_bytes(1, D, ps), dtype=torch.uint8, device=DEV)
    k, v = normal((1, 1, 16, D), 1, torch.bfloat16), normal((1, 1, 16, D), 2, torch.bfloat16)
    L.loma_kv4_append(k, v, pool, di32([[n - 1]]), ps, di32([0]))
    kc, vc = torch.zeros_like(k), torch.zeros_like(v)
    L.loma_kv4_load(pool, di32([[n - 1]]), ps, di32([16]), kc, vc)
    assert np.array_equal(npf(kc), stored(k, torch.bfloat16)) and np.array_equal(npf(vc), stored(v, torch.bfloat16))
    for dtype, flags in KINDS:
        s = dict(q=normal((1, 2, 1, D), 3, dtype), kt=normal((1, 1, 1, D), 4, dtype), vt=normal((1, 1, 1, D), 5, dtype))
        o = torch.zeros(1, 2, 1, D, dtype=dtype, device=DEV)
        ws = torch.empty(L.loma_decode_kv4_workspace_bytes(1, 2, 1, D, 16, 0), dtype=torch.uint8, device=DEV)
        L.loma_decode_attn_kv4(s["q"], None, None, s["kt"], s["vt"], di32([0]), 0, pool, di32([[n - 1]]), ps, di32([16]), 16, o, None, workspace=ws, flags=flags)
        want, _, o_abs = C.decode_attn_kv4(npf(s["q"])[:, :, 0], [C.kv4_values(npf(k[0]))], [C.kv4_values(npf(v[0]))], [npf(s["kt"][0])], [npf(s["vt"][0])])
        assert (np.abs(npf(o)[:, :, 0] - want) <= 2.0**-7 * o_abs + 1e-6).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_row_by_row_in_any_order(dtype, D):
    """Rows share words with their neighbours: entry after entry, in any order and in pieces, the pool becomes what one call makes it."""
    B, Hkv, ps, n = 3, 2, 16, 45
    k, v = normal((B, Hkv, n, D), 1, dtype), normal((B, Hkv, n, D), 2, dtype)
    table, whole = table_of(B, 3, 0), new_pool(11, Hkv, D, ps, 255)
    L.loma_kv4_append(k, v, whole, table, ps, di32([0] * B))
    rng = np.random.default_rng(0)
    single, pieces = new_pool(11, Hkv, D, ps, 255), new_pool(11, Hkv, D, ps, 255)
    for e in rng.permutation(n).tolist():
        L.loma_kv4_append(k[:, :, e:e + 1], v[:, :, e:e + 1], single, table, ps, di32([e] * B))
    cuts = [0, 1, 4, 5, 11, 18, 33, 44, n]
    for e0, e1 in rng.permutation(list(zip(cuts, cuts[1:]))).tolist():
        L.loma_kv4_append(k[:, :, e0:e1], v[:, :, e0:e1], pieces, table, ps, di32([e0] * B))
    assert torch.equal(single, whole) and torch.equal(pieces, whole)


# ------------------------------------------------------------------------------------------------ decode
def make(B, Hq, Hkv, D, mems, tails, ps, dtype, seed=0, cap=None, std=1.0, garbage=True):
    """A batch: memory entries stored through the block table, tails in caches; everything no request may see is NaN."""
    top, most = max(max(mems), 0), max(max(tails), 0)
    cap = most + 1 if cap is None else cap
    M = -(-top // ps) + 1
    table = table_of(B, M, seed)
    pool = new_pool(B * M + 2, Hkv, D, ps, 255 if garbage else 0)
    k, v = (normal((B, Hkv, max(top, 1), D), seed + 1 + i, dtype, std) for i in (0, 1))
    L.loma_kv4_append(k, v, pool, table, ps, di32([0] * B), di32(mems))
    kt, vt = (normal((B, Hkv, cap, D), seed + 3 + i, dtype, std) for i in (0, 1))
    for b, n in enumerate(tails):
        kt[b, :, max(n, 0):], vt[b, :, max(n, 0):] = float("nan"), float("nan")
    s = dict(B=B, Hq=Hq, Hkv=Hkv, D=D, ps=ps, dtype=dtype, mems=list(mems), tails=list(tails), max_mem=top, max_tail=most, table=table, pool=pool, k=k, v=v, kt=kt, vt=vt,
             kn=normal((B, Hkv, 1, D), seed + 5, dtype, std), vn=normal((B, Hkv, 1, D), seed + 6, dtype, std), q=normal((B, Hq, 1, D), seed + 7, dtype, std),
             o=torch.full((B, Hq, 1, D), 7.0, dtype=dtype, device=DEV), lse=torch.full((B, Hq), 7.0, device=DEV))
    s["ws"] = torch.full((L.loma_decode_kv4_workspace_bytes(B, Hq, Hkv, D, top, most),), 255, dtype=torch.uint8, device=DEV)
    return s


def call(s, flags=0, scale=0.0, token=True, **over):
    a = {**s, **over}
    L.loma_decode_attn_kv4(a["q"], a["kn"] if token else None, a["vn"] if token else None, a["kt"], a["vt"], di32(a["tails"]), a["max_tail"], a["pool"], a["table"],
                           a["ps"], di32(a["mems"]), a["max_mem"], a["o"], a["lse"], workspace=a["ws"], flags=flags, softmax_scale=scale)


def expected(s, scale=None, mems=None, tails=None):
    mems, tails = mems or s["mems"], tails or s["tails"]
    kv, vv = C.kv4_values(npf(s["k"])), C.kv4_values(npf(s["v"]))
    km, vm = ([x[b, :, : max(n, 0)] for b, n in enumerate(mems)] for x in (kv, vv))
    kt, vt = [], []
    for out, cache, new in ((kt, s["kt"], s["kn"]), (vt, s["vt"], s["vn"])):
        c, x = npf(cache), npf(new)
        out += [None if n < 0 else np.concatenate([c[b, :, :n], x[b]], 1) for b, n in enumerate(tails)]
    q = npf(s["q"])[:, :, 0]
    o, lse, o_abs = C.decode_attn_kv4(q, km, vm, kt, vt, scale)
    reach = np.zeros(lse.shape)
    g = s["Hq"] // s["Hkv"]
    for b, n in enumerate(tails):
        for hq in range(s["Hq"]):
            if n >= 0:
                keys = np.concatenate([km[b][hq // g], kt[b][hq // g]])
                reach[b, hq] = (np.abs(keys) @ np.abs(q[b, hq])).max() * (s["D"]**-0.5 if scale is None else scale)
    return o, lse, o_abs, reach


def tolerances(s, o, o_abs, reach, flags):
    n = s["max_mem"] + s["max_tail"] + 1
    score = (s["D"] + 8) * 2.0**-23 * reach
    soft = (2 * score + n * 2.0**-23 + 2.0**-20)[..., None] * o_abs
    if s["dtype"] == torch.float32:
        return soft + 2.0**-24 * np.abs(o), score + n * 2.0**-23 + 2.0**-20 * (1 + reach)
    return soft + 2.0**-8 * np.abs(o) + (0 if flags else 2.0**-8 * o_abs), score + n * 2.0**-23 + 2.0**-20 * (1 + reach)


def check(s, flags=0, scale=None, before=None, **kw):
    o, lse, o_abs, reach = expected(s, scale, **kw)
    tails = kw.get("tails") or s["tails"]
    t_o, t_l = tolerances(s, o, o_abs, reach, flags)
    live = [b for b, n in enumerate(tails) if n >= 0]
    idle = [b for b, n in enumerate(tails) if n < 0]
    go, gl = npf(s["o"])[:, :, 0], npf(s["lse"])
    assert np.isfinite(go[live]).all() and np.isfinite(gl[live]).all()
    assert (np.abs(go - o)[live] <= t_o[live]).all(), float((np.abs(go - o)[live] / t_o[live]).max())
    assert (np.abs(gl - lse)[live] <= t_l[live]).all(), float((np.abs(gl - lse)[live] / t_l[live]).max())
    assert (go[idle] == 7.0).all() and (gl[idle] == 7.0).all()


CASES = [
    # B, Hq, Hkv, D, mems, tails, ps
    (1, 1, 1, 64, [0], [0], 16),
    (1, 1, 1, 128, [1], [0], 16),
    (1, 3, 1, 128, [16], [15], 16),
    (2, 8, 2, 64, [17, 0], [16, 1], 16),
    (3, 8, 8, 128, [31, 32, 33], [0, 63, 64], 32),
    (4, 12, 3, 64, [15, 100, 64, 1], [5, -1, 40, 0], 64),
    (5, 40, 4, 128, [200, 0, 47, 48, 49], [3, 17, -1, -1, 90], 16),
    (2, 24, 2, 64, [300, 513], [33, 2], 128),
    (2, 18, 1, 128, [1000, 999], [0, 20], 256),
    (7, 6, 6, 64, [0, 0, 0, 0, 0, 0, 0], [0, 1, 15, 16, 17, 31, -1], 16),
    (1, 8, 8, 128, [5000], [10], 16),
    (33, 4, 2, 128, [(37 * b) % 700 for b in range(33)], [(b * 7) % 50 - 1 for b in range(33)], 64),
    (600, 2, 2, 64, [(13 * b) % 90 for b in range(600)], [(b * 5) % 20 - 2 for b in range(600)], 16),
    (1, 32, 1, 64, [3000], [100], 32),
]


@pytest.mark.parametrize("dtype,flags", KINDS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_decode(case, dtype, flags):
    s = make(*CASES[case], dtype, seed=10 * case)
    kt, vt = s["kt"].clone(), s["vt"].clone()
    call(s, flags)
    check(s, flags)
    for b, n in enumerate(s["tails"]):            # the new token is stored, everything else stays
        if n >= 0:
            kt[b, :, n], vt[b, :, n] = s["kn"][b, :, 0], s["vn"][b, :, 0]
    for got, want in ((s["kt"], kt), (s["vt"], vt)):
        assert np.array_equal(npf(got), npf(want), equal_nan=True)


CUT = [
    (2, 24, 2, 128, [3000, 517], [40, 0], 16),
    (3, 8, 8, 64, [1700, 0, 333], [-1, 17, 5], 32),
    (1, 40, 2, 64, [2100], [3], 128),
    (5, 6, 3, 128, [0, 31, 32, 33, 900], [0, 15, 16, 31, 100], 16),
    (2, 17, 1, 128, [64, 4000], [100, 1], 256),
]


@pytest.mark.parametrize("dtype,flags", KINDS)
@pytest.mark.parametrize("case", range(len(CUT)))
def test_decode_cut_into_equal_shares(case, dtype, flags):
    """Bounds as high as a table's capacity: units are cut among all workers, and joined from the workspace."""
    s = make(*CUT[case], dtype, seed=100 + case)
    s["table"] = torch.cat([s["table"], torch.full((s["B"], 200000 // s["ps"]), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    top, s["max_mem"] = s["max_mem"], 150000
    s["ws"] = torch.full((L.loma_decode_kv4_workspace_bytes(s["B"], s["Hq"], s["Hkv"], s["D"], 150000, s["max_tail"]),), 255, dtype=torch.uint8, device=DEV)
    call(s, flags)
    s["max_mem"] = top
    check(s, flags)


@pytest.mark.parametrize("B,Hq,Hkv,D,most,ps", [(75, 16, 8, 128, 300, 16), (150, 20, 4, 64, 500, 64), (70, 9, 9, 128, 90, 16)])
def test_decode_many_units(B, Hq, Hkv, D, most, ps):
    """More units than run at once: cut, rows joined by one set of lanes each; and short ones, whole."""
    s = make(B, Hq, Hkv, D, [(37 * b) % most for b in range(B)], [(b * 7) % 40 - 1 for b in range(B)], ps, torch.bfloat16, seed=B)
    call(s)
    check(s)


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_token_already_stored_own_scale_no_lse(dtype, flags):
    s = make(3, 8, 2, 128, [70, 0, 333], [20, 3, -1], 32, dtype)
    for b, n in enumerate(s["tails"]):
        if n >= 0:
            s["kt"][b, :, n], s["vt"][b, :, n] = s["kn"][b, :, 0], s["vn"][b, :, 0]
    kt = s["kt"].clone()
    call(s, flags, 0.31, token=False)
    check(s, flags, 0.31)
    assert np.array_equal(npf(s["kt"]), npf(kt), equal_nan=True)
    o = s["o"].clone()
    s["o"].fill_(7.0)
    call(s, flags, 0.31, token=False, lse=None)
    assert torch.equal(s["o"], o)


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_lengths_outside_the_bounds(dtype, flags):
    s = make(4, 4, 2, 64, [100, 60, 40, 90], [12, 30, 7, 30], 16, dtype)
    s["max_mem"], s["max_tail"] = 64, 20
    s["kt"], s["vt"] = s["kt"].nan_to_num(0.5), s["vt"].nan_to_num(0.5)
    call(s, flags, tails=[12, 2**31 - 1, 7, 30], mems=[100, 60, -3, 2**31 - 1])
    check(s, flags, mems=[64, 60, 0, 64], tails=[12, 20, 7, 20])


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_without_a_pool(dtype, flags):
    s = make(2, 4, 2, 128, [0, 0], [40, 3], 16, dtype)
    call(s, flags, pool=None, table=None)
    check(s, flags)


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_under_high_bounds_and_all_idle(dtype, flags):
    s = make(3, 8, 2, 64, [40, 0, 7], [-1, 4, 0], 16, dtype, cap=2000)
    s["max_tail"] = 1999
    s["table"] = torch.cat([s["table"], torch.full((3, 4000), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    s["max_mem"] = s["table"].shape[1] * 16
    s["ws"] = torch.empty(L.loma_decode_kv4_workspace_bytes(3, 8, 2, 64, s["max_mem"], 1999), dtype=torch.uint8, device=DEV)
    call(s, flags)
    s["max_mem"] = 40
    check(s, flags)
    s["o"].fill_(7.0), s["lse"].fill_(7.0)
    call(s, flags, tails=[-1, -5, -2**31])
    assert (s["o"] == 7.0).all() and (s["lse"] == 7.0).all()


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_sharp_scores(dtype, flags):
    """The softmax reference moves many times along a sequence: scores that rise by hundreds, and weights on a few entries."""
    s = make(2, 4, 2, 128, [900, 2000], [40, 3], 16, dtype, std=4.0)
    rise = torch.linspace(0, 6, s["k"].shape[2], device=DEV)[None, None, :, None]
    s["k"] = (s["k"] * rise).to(dtype)
    L.loma_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["ps"], di32([0, 0]), di32(s["mems"]))
    call(s, flags)
    check(s, flags)


@pytest.mark.parametrize("dtype,flags", KINDS)
@pytest.mark.parametrize("std_q,std_v", [(1e-6, 1e-6), (1.0, 1e6), (1e3, 1e-12)])
def test_decode_small_and_large_numbers(std_q, std_v, dtype, flags):
    s = make(2, 4, 2, 64, [100, 37], [20, 3], 16, dtype)
    s["q"] = (s["q"] * std_q).to(dtype)
    for x in ("v", "vt", "vn"):
        s[x] = (s[x] * std_v).to(dtype)
    L.loma_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["ps"], di32([0, 0]), di32(s["mems"]))
    call(s, flags)
    check(s, flags)


@pytest.mark.parametrize("dtype,flags", KINDS)
@pytest.mark.parametrize("where", ["memory k", "memory v", "tail k", "tail v", "token k", "query"])
@pytest.mark.parametrize("n", [40, 700])
def test_decode_nan_reaches_the_outputs_of_its_sequence_alone(n, where, dtype, flags):
    s = make(3, 8, 2, 128, [n, n, n], [20, 20, 20], 16, dtype)
    which, x = where.split(" ") if " " in where else (where, "")
    if which == "memory":
        s[x][1, 1, n // 2, 3] = float("nan")
        L.loma_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["ps"], di32([0] * 3), di32(s["mems"]))
    elif which == "tail":
        s[x + "t"][1, 1, 7, 3] = float("nan")
    elif which == "token":
        s["kn"][1, 1, 0, 3] = float("nan")
    else:
        s["q"][1, 5, 0, 3] = float("nan")
    call(s, flags)
    o = npf(s["o"])[:, :, 0]
    assert np.isfinite(o[[0, 2]]).all() and np.isfinite(o[1, :4]).all()
    if x == "v":                                  # a value: its feature, or its group of 32 in memory
        bad = np.isnan(o[1, 4:])
        assert bad[:, 3].all() and bad[:, :32].all() == (which == "memory") and not bad[:, 32:].any()
    elif which == "query":
        assert np.isnan(o[1, 5]).all() and np.isfinite(o[1, [4, 6, 7]]).all()
    else:
        assert np.isnan(o[1, 4:]).all()
    if x != "v":
        assert np.isnan(npf(s["lse"])[1, 5])


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_infinite_tail_values_at_the_end_of_a_block(dtype, flags):
    """The last block repeats the row of the new token where it reads past the end: an infinite value there counts once."""
    s = make(2, 4, 2, 64, [40, 10], [4, 18], 16, dtype)
    s["vn"][0, 0, 0, 5] = float("inf")
    s["vt"][1, 1, 17, 9] = float("-inf")
    call(s, flags)
    o, want = npf(s["o"])[:, :, 0], expected(s)[0]
    assert np.array_equal(np.isinf(o), np.isinf(want)) and np.isinf(o).sum() == 4 and not np.isnan(o).any()


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_scores_of_minus_infinity_have_no_weight(dtype, flags):
    s = make(1, 2, 1, 64, [600], [40], 16, dtype)
    s["q"].abs_()
    s["kt"][0, 0, :20] = float("-inf")            # whole blocks, and parts of them, without weight
    call(s, flags)
    want = C.decode_attn_kv4(npf(s["q"])[:, :, 0], [C.kv4_values(npf(s["k"][0]))], [C.kv4_values(npf(s["v"][0]))],
                             [np.concatenate([npf(s["kt"][0])[:, 20:40], npf(s["kn"][0])], 1)], [np.concatenate([npf(s["vt"][0])[:, 20:40], npf(s["vn"][0])], 1)])
    assert (np.abs(npf(s["o"])[:, :, 0] - want[0]) <= 2.0**-6 * want[2]).all()


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_page_numbers_out_of_range_stay_in_the_pool(dtype, flags):
    s = make(3, 4, 2, 64, [60, 60, 60], [3, 3, 3], 16, dtype, garbage=False)
    bad = s["table"].clone()
    bad[0, 1], bad[0, 2], bad[2, 0] = -1, 2**31 - 1, -(2**31)
    n = s["pool"].shape[0]
    call(s, flags, table=bad)
    got = [s["o"].clone(), s["lse"].clone()]
    s["kt"][:, :, 3], s["vt"][:, :, 3] = float("nan"), float("nan")
    call(s, flags, table=bad.clamp(0, n - 1))
    assert torch.equal(got[0], s["o"]) and torch.equal(got[1], s["lse"])


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_repeats_and_runs_beside_itself(dtype, flags):
    """The same bits again, and from two streams at once with workspaces of their own."""
    sets = [make(6, 8, 2, 128, [(j * 300 + 77 * b) % 1500 for b in range(6)], [5 * b for b in range(6)], 16, dtype, seed=50 * j) for j in (1, 2)]
    for s in sets:
        call(s, flags)
    first = [(s["o"].clone(), s["lse"].clone()) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s in sets:
            s["o"].fill_(7.0)
        torch.cuda.synchronize()
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                call(s, flags)
        torch.cuda.synchronize()
        for s, (o, lse) in zip(sets, first):
            assert torch.equal(s["o"], o) and torch.equal(s["lse"], lse)


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_replayed_with_other_lengths(dtype, flags):
    s = make(4, 8, 2, 64, [500, 300, 200, 90], [30, 30, 30, 30], 16, dtype)
    s["kt"], s["vt"] = s["kt"].nan_to_num(0.25), s["vt"].nan_to_num(0.25)
    tails, mems = di32([1, 2, 3, 4]), di32([10, 0, 20, 30])

    def step():
        L.loma_decode_attn_kv4(s["q"], s["kn"], s["vn"], s["kt"], s["vt"], tails, 30, s["pool"], s["table"], 16, mems, 500, s["o"], s["lse"], workspace=s["ws"], flags=flags)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for m, t in (([500, 300, 200, 90], [30, 0, 12, 5]), ([0, 1, 17, 90], [3, -1, 16, 30]), ([33, 300, 0, 5], [0, 0, 0, 29])):
        kt, vt = s["kt"].clone(), s["vt"].clone()
        s["o"].fill_(7.0), s["lse"].fill_(7.0)
        mems.copy_(di32(m)), tails.copy_(di32(t))
        graph.replay()
        torch.cuda.synchronize()
        check({**s, "kt": kt, "vt": vt}, flags, mems=m, tails=t)


def test_decode_refuses_what_it_cannot_take():
    s = make(2, 4, 2, 64, [20, 20], [3, 3], 16, torch.bfloat16)
    with pytest.raises(L.LomaError):
        call(s, max_tail=s["kt"].shape[2])
    with pytest.raises(L.LomaError):
        call(s, ws=s["ws"][: 16])
    with pytest.raises(ValueError):
        call(s, q=s["q"].half())
    with pytest.raises(ValueError):
        call(s, pool=s["pool"][:, :-16].contiguous())
    with pytest.raises(ValueError):
        call(s, kt=s["kt"].cpu())
    with pytest.raises(L.LomaError):
        call(s, ps=8)


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_generation_with_memory_in_4_bits(dtype):
    """LoMA's loop over 4-bit memory for a batch whose sequences stand at different points of their chunks: decode steps; a full tail is
    compressed (loma_compress_step_ragged over the tail alone), its t memory rows are stored in 4 bits behind pages drawn by
    loma_paged_extend; one sequence branches off another; one ends and gives its pages back; the pool is compacted.  Every step against
    the oracle, from the state the device keeps."""
    B, Hh, D, c, t, ps, M = 4, 3, 64, 4, 4, 16, 3
    tc, n_pages = c * t, 14
    rng = np.random.default_rng(0)
    e = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
    table, held, refs, free, taken = e(B, M).fill_(-1), di32([0] * B), di32([0] * n_pages), di32(rng.permutation(n_pages)), di32([0])
    mems, tails = di32([0] * B), di32([5, 0, 12, -1])
    pool = new_pool(n_pages, Hh, D, ps, 255)
    kt, vt = (normal((B, Hh, tc + 1, D), 1 + i, dtype) for i in (0, 1))
    ws = torch.empty(L.loma_decode_kv4_workspace_bytes(B, Hh, Hh, D, M * ps, tc), dtype=torch.uint8, device=DEV)
    rs, pg, counts = e(B + 1), e(B + 1), e(4)
    memory = [[np.zeros((Hh, 0, D)) for _ in range(B)] for _ in "kv"]       # what the memory entries stand for
    tol = 2.0**-7 if dtype == torch.bfloat16 else 1e-5
    for step in range(110):
        q, kn, vn = (normal((B, Hh, 1, D), 100 + 10 * step + i, dtype) for i in range(3))
        o = torch.zeros(B, Hh, 1, D, dtype=dtype, device=DEV)
        at = tails.tolist()
        L.loma_decode_attn_kv4(q, kn, vn, kt, vt, tails, tc, pool, table, ps, mems, M * ps, o, None, workspace=ws)
        tail = [[None if n < 0 else npf(x)[b, :, : n + 1] for b, n in enumerate(at)] for x in (kt, vt)]
        want, _, o_abs = C.decode_attn_kv4(npf(q)[:, :, 0], memory[0], memory[1], tail[0], tail[1])
        live = [b for b, n in enumerate(at) if n >= 0]
        assert (np.abs(npf(o)[:, :, 0] - want)[live] <= tol * (o_abs + np.abs(want))[live] + 1e-6).all(), step
        tails.add_((tails >= 0).to(torch.int32))
        full = tails == tc
        if bool(full.any()):
            qm, km, vm = (normal((B, Hh, t, D), 5000 + 10 * step + i, dtype) for i in range(3))
            om = torch.zeros(B, Hh, t, D, dtype=dtype, device=DEV)
            which = torch.where(full, 0, -1).to(torch.int32)
            before = [npf(kt), npf(vt)]
            L.loma_compress_step_ragged(qm, km, vm, kt, vt, om, None, which, 0, c, t)
            new = torch.where(full, t, 0).to(torch.int32)
            L.loma_paged_extend(torch.where(full, mems, -1).to(torch.int32), new, held, None, free, taken, table, ps, rs, pg, held, e(0), e(0), e(0))
            L.loma_kv4_append(kt[:, :, :t], vt[:, :, :t], pool, table, ps, torch.where(full, mems, -1).to(torch.int32), new)
            for b in full.nonzero().flatten().tolist():
                wo, _, wk, wv = O.compress_step(npf(qm)[b:b + 1], npf(km)[b:b + 1], npf(vm)[b:b + 1], before[0][b:b + 1], before[1][b:b + 1], 0, c, t)
                assert (np.abs(npf(om)[b] - wo[0]) <= 2 * tol * (1 + np.abs(wo[0]))).all()
                for m, x in zip(memory, (km, vm)):
                    m[b] = np.concatenate([m[b], C.kv4_values(npf(x)[b])], 1)
            mems.add_(new)
            tails.copy_(torch.where(full, 0, tails))
            assert int(pg[-1]) <= n_pages
        if step == 76:                             # slot 3 goes on from sequence 0: whole pages shared, the last one copied
            par = di32([0, 1, 2, 0])
            out, lo, ho, src, dst = e(B, M), e(B), e(B), e(8), e(8)
            fws = torch.empty(L.loma_paged_fork_workspace_bytes(B), dtype=torch.uint8, device=DEV)
            L.loma_paged_fork(par, mems, None, held, table, ps, out, lo, ho, refs, free, taken, src, dst, counts, workspace=fws)
            L.loma_paged_copy([pool], src, dst, counts[:1])
            assert counts.tolist()[0] == 1 and refs.tolist().count(1) == 1
            table, held, mems = out, ho, lo.clamp(min=0)
            kt[3], vt[3] = kt[0], vt[0]
            tails[3] = tails[0]
            for m in memory:
                m[3] = m[0].copy()
        if step == 90:                             # sequence 2 ends
            L.loma_paged_release(di32([-1, -1, 0, -1]), held, table, ps, held, refs, free, taken, counts)
            tails[2], mems[2] = -1, 0
            for m in memory:
                m[2] = np.zeros((Hh, 0, D))
            assert counts.tolist()[1] > 0
        if step == 100:
            pm, src, dst = e(n_pages), e(n_pages), e(n_pages)
            L.loma_paged_compact(held, table, refs, free, taken, pm, src, dst, counts)
            L.loma_paged_copy([pool], src, dst, counts[:1])
            used = {p for row, h in zip(table.tolist(), held.tolist()) for p in row[:h]}
            assert used == set(range(len(used)))
    assert mems.tolist()[0] > ps and mems.tolist()[3] > ps      # shared pages and copied ones were both in use


def test_bookkeeping_and_decode_captured_together():
    """Extend, append, decode, fork, copy, release in one captured graph, replayed from the same start: the same results as eager."""
    B, Hq, Hkv, D, ps, M, n_pages, dtype = 4, 4, 2, 64, 16, 6, 40, torch.bfloat16
    e = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    inputs = [normal((B, Hkv, 20, D), 1, dtype), normal((B, Hkv, 20, D), 2, dtype), normal((B, Hq, 1, D), 3, dtype), normal((B, Hkv, 1, D), 4, dtype)]

    def fresh():
        s = dict(table=e(B, M) - 1, held=e(B), refs=e(n_pages), free=di32(np.arange(n_pages)[::-1].copy()), taken=e(1), mems=di32([0, 0, 0, -1]), out=e(B, M), lo=e(B), ho=e(B),
                 src=e(30), dst=e(30), counts=e(4), c2=e(4), rs=e(B + 1), pg=e(B + 1), sl=e(60), sq=e(60), po=e(60), pool=new_pool(n_pages, Hkv, D, ps),
                 kt=torch.zeros(B, Hkv, 4, D, dtype=dtype, device=DEV), vt=torch.zeros(B, Hkv, 4, D, dtype=dtype, device=DEV), tails=di32([0, 1, 2, 3]),
                 o=torch.zeros(B, Hq, 1, D, dtype=dtype, device=DEV))
        s["kt"], s["vt"] = normal((B, Hkv, 4, D), 8, dtype), normal((B, Hkv, 4, D), 9, dtype)
        return s

    ws = torch.empty(L.loma_decode_kv4_workspace_bytes(B, Hq, Hkv, D, M * ps, 3), dtype=torch.uint8, device=DEV)
    fws = torch.empty(L.loma_paged_fork_workspace_bytes(B), dtype=torch.uint8, device=DEV)
    new, par, keep = di32([20, 7, 13, 5]), di32([0, 0, 2, 1]), di32([16, -1, 3, 0])

    def step(s):
        L.loma_paged_extend(s["mems"], new, s["held"], None, s["free"], s["taken"], s["table"], ps, s["rs"], s["pg"], s["held"], s["sl"], s["sq"], s["po"])
        L.loma_kv4_append(inputs[0], inputs[1], s["pool"], s["table"], ps, s["mems"], new)
        s["mems"].add_(torch.where(s["mems"] >= 0, new, 0))
        L.loma_paged_fork(par, s["mems"], None, s["held"], s["table"], ps, s["out"], s["lo"], s["ho"], s["refs"], s["free"], s["taken"], s["src"], s["dst"], s["counts"], workspace=fws)
        L.loma_paged_copy([s["pool"]], s["src"], s["dst"], s["counts"][:1])
        L.loma_decode_attn_kv4(inputs[2], inputs[3], inputs[3], s["kt"], s["vt"], s["tails"], 3, s["pool"], s["out"], ps, s["lo"], M * ps, s["o"], None, workspace=ws)
        L.loma_paged_release(keep, s["ho"], s["out"], ps, s["ho"], s["refs"], s["free"], s["taken"], s["c2"])

    eager = fresh()
    step(eager)
    assert eager["lo"].tolist() == [20, 20, 13, 7] and eager["counts"].tolist()[0] == 1 and eager["c2"].tolist()[1] > 0
    s = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    for _ in range(2):
        for k, v in fresh().items():
            s[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for k in s:
            assert torch.equal(s[k], eager[k]), k


def test_prompt_memory_through_load_and_prefill():
    """A prompt's memory in 4 bits, read back for the next piece of a prompt: loma_prefill_attn_ragged over what the entries stand for."""
    B, Hh, D, ps, l, dtype = 3, 2, 128, 16, 12, torch.bfloat16
    mems, cap = [40, 0, 23], 80
    k, v = normal((B, Hh, 40, D), 1, dtype), normal((B, Hh, 40, D), 2, dtype)
    pool, table = new_pool(12, Hh, D, ps, 255), table_of(B, 3, 0)
    L.loma_kv4_append(k, v, pool, table, ps, di32([0] * B), di32(mems))
    kc, vc = (torch.zeros(B, Hh, cap, D, dtype=dtype, device=DEV) for _ in "kv")
    L.loma_kv4_load(pool, table, ps, di32(mems), kc, vc)
    q, kn, vn = (normal((B, Hh, l, D), 3 + i, dtype) for i in range(3))
    o = torch.zeros_like(q)
    hk, hv = npf(kc), npf(vc)
    L.loma_prefill_attn_ragged(q, kn, vn, kc, vc, o, None, di32(mems), 40)
    for b, n in enumerate(mems):
        assert np.array_equal(hk[b, :, :n], stored(k, dtype)[b, :, :n])
        want = O.prefill_attn(npf(q)[b:b + 1], npf(kn)[b:b + 1], npf(vn)[b:b + 1], hk[b:b + 1], hv[b:b + 1], n)[0]
        assert (np.abs(npf(o)[b] - want[0]) <= 2e-2).all()



FIRST_CALL = """
import sys
import torch
from paper_2401_09486_b200 import binding as L
d, bf, which = "cuda:0", torch.bfloat16, sys.argv[1]
i = lambda *x: torch.tensor(x, dtype=torch.int32, device=d)
z = lambda *x: torch.zeros(x, dtype=torch.int32, device=d)
k, q = torch.randn(2, 2, 20, 64, device=d).to(bf), torch.randn(2, 4, 1, 64, device=d).to(bf)
kn, vn, o = k[:, :, :1].contiguous(), k[:, :, 1:2].contiguous(), torch.zeros_like(q)
kc, vc = torch.zeros_like(k), torch.zeros_like(k)
pool = torch.zeros(8, L.loma_kv4_page_bytes(2, 64, 16), dtype=torch.uint8, device=d)
some = torch.randint(1, 100, tuple(pool.shape), dtype=torch.uint8, device=d)
ws = torch.zeros(1 << 24, dtype=torch.uint8, device=d)
table, wide, long = i(0, 1, 2, 3).view(2, 2), torch.cat([i(0, 1, 2, 3).view(2, 2), z(2, 20000)], 1).contiguous(), z(400, 3)
lens, tails, held, refs, free, taken, counts, src, dst = i(20, 7), i(3, 0), i(2, 2), z(8), i(7, 6, 5, 4), i(1), z(4), z(6), z(6)
out, wide_out, l2, h2, l4, h4, none, one4, page_map = z(2, 2), z(400, 3), z(2), z(2), z(400), z(400), z(400) - 1, z(400) + 1, z(8)
state = (refs, free, taken)
parents, keep, keep4, one, zero = i(1, 0), z(2), z(400), i(1), i(0)
decode = lambda bound: L.loma_decode_attn_kv4(q, kn, vn, kc, vc, tails, 3, pool, wide, 16, lens, bound, o, None, workspace=ws)
calls = {
    "append": (pool, lambda: L.loma_kv4_append(k, k, pool, table, 16, keep)),
    "load": (kc, lambda: L.loma_kv4_load(some, table, 16, lens, kc, vc)),
    "whole": (o, lambda: decode(32)), "cluster": (o, lambda: decode(1000)), "cut": (o, lambda: decode(300000)),
    "release": (counts, lambda: L.loma_paged_release(keep, held, table, 16, held, *state, counts)),
    "release_long": (counts, lambda: L.loma_paged_release(keep4, one4, long, 16, one4, *state, counts)),
    "fork": (out, lambda: L.loma_paged_fork(parents, lens, None, held, table, 16, out, l2, h2, *state, src, dst, counts, workspace=ws)),
    "fork_long": (counts, lambda: L.loma_paged_fork(none, one4, None, one4, long, 16, wide_out, l4, h4, *state, src, dst, counts, workspace=ws)),
    "compact": (page_map, lambda: L.loma_paged_compact(held, table, *state, page_map, src, dst, counts)),
    "compact_long": (page_map, lambda: L.loma_paged_compact(one4, long, *state, page_map, src, dst, counts)),
    "copy": (pool, lambda: L.loma_paged_copy([pool, some], one, zero, one)),
}
if which == "copy":
    pool[1] = 1
result, call = calls[which]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
graph.replay()
torch.cuda.synchronize()
assert result.ne(0).any() and (which != "copy" or bool((pool[0] == 1).all()))
print("captured")
"""


@pytest.mark.parametrize("which", ["append", "load", "whole", "cluster", "cut", "release", "release_long", "fork", "fork_long", "compact", "compact_long", "copy"])
def test_the_first_call_of_a_process_may_be_captured(which):
    out = subprocess.run([sys.executable, "-c", FIRST_CALL, which], capture_output=True, text=True, timeout=300, cwd=build.ROOT)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]


# ------------------------------------------------------------------------------------------------ calls between others
@pytest.mark.parametrize("dtype,flags", KINDS)
@pytest.mark.parametrize("B,live", [(300, {0, 31, 32, 65, 298}), (300, {299}), (97, {0}), (64, {5, 38, 63}), (1100, {3, 600, 1098})])
def test_decode_few_requests_in_many_slots(B, live, dtype, flags):
    """Workers pass over the slots without a request, in runs of any length and past the batch's end, cut and whole."""
    s = make(B, 6, 2, 64, [40 + b % 50 if b in live else 9 for b in range(B)], [b % 33 if b in live else -1 - b % 3 for b in range(B)], 16, dtype, seed=B)
    call(s, flags)
    check(s, flags)
    s["table"] = torch.cat([s["table"], torch.full((B, 2000), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    top, s["max_mem"] = s["max_mem"], 30000
    s["ws"] = torch.full((L.loma_decode_kv4_workspace_bytes(B, 6, 2, 64, 30000, s["max_tail"]),), 255, dtype=torch.uint8, device=DEV)
    for b in range(B):
        if b not in live:
            continue
        s["kt"][b, :, s["tails"][b]:], s["vt"][b, :, s["tails"][b]:] = float("nan"), float("nan")
    s["o"].fill_(7.0), s["lse"].fill_(7.0)
    call(s, flags)
    s["max_mem"] = top
    check(s, flags)


@pytest.mark.parametrize("before", ["memcpy", "memset", "event", "torch", "nothing"])
def test_copy_behind_other_work(before):
    """The copy may be launched early behind a kernel; behind anything else it waits all the same, eager and captured."""
    pool = torch.randint(0, 256, (9, 1 << 20), dtype=torch.uint8, device=DEV)
    lists, ready, start = di32([[0, 3, 5], [1, 2, 4]]), di32([[0, 3, 5], [1, 2, 4]]), pool.clone()
    n, other, big = di32([3]), torch.cuda.Stream(), torch.empty(1 << 27, dtype=torch.uint8, device=DEV)
    want = start.clone()
    want[[1, 2, 4]] = start[[0, 3, 5]]

    def step():
        now = torch.cuda.current_stream()
        if before == "memcpy":
            pool.copy_(start)
            lists.copy_(ready)
        elif before == "memset":
            big.zero_()
        elif before == "event":                    # lists and pool made on another stream, behind 128 MB of other writes
            other.wait_stream(now)
            with torch.cuda.stream(other):
                big.fill_(3)
                pool.copy_(start)
                lists.copy_(ready)
            now.wait_stream(other)
        elif before == "torch":
            torch.add(ready, 0, out=lists)
        L.loma_paged_copy([pool], lists[0], lists[1], n)

    def reset():
        pool.copy_(start)
        if before in ("memcpy", "event"):
            pool.zero_()
        if before in ("memcpy", "event", "torch"):
            lists.fill_(-1)
        torch.cuda.synchronize()

    for _ in range(3):
        reset()
        step()
        assert torch.equal(pool, want)
    reset()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want)


def test_calls_from_two_threads_at_once():
    """Threads with streams, workspaces and lists of their own: the results of calls made alone."""
    sets = [make(5, 8, 2, 128, [(j * 900 + 77 * b) % 1500 for b in range(5)], [5 * b for b in range(5)], 16, torch.bfloat16, seed=90 + j) for j in range(4)]
    for s in sets:
        call(s)
    want = [(s["o"].clone(), s["lse"].clone()) for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(s, o, lse, j):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                s["o"].fill_(7.0), s["lse"].fill_(7.0)
                call(s)
                pool = torch.arange(12, device=DEV, dtype=torch.int32).repeat(64, 1).t().contiguous().view(torch.uint8)
                table, held, refs, free, taken, counts = di32([[0, 1, 2], [3, 4, 5]]), di32([3, 3]), di32([0] * 12), di32(list(range(12))), di32([6]), di32([0] * 4)
                L.loma_paged_release(di32([16 * j % 48, -1]), held, table, 16, held, refs, free, taken, counts)
                L.loma_paged_copy([pool], di32([7]), di32([8]), di32([1]))
                stream.synchronize()
                kept = min(j, 3) if j < 3 else 0
                if not (torch.equal(s["o"], o) and torch.equal(s["lse"], lse)) or held.tolist() != [kept, 3] or int(taken) != 6 - (3 - kept) or not torch.equal(pool[8], pool[7]):
                    wrong.append(j)

    import threading
    threads = [threading.Thread(target=work, args=(s, *w, j)) for j, (s, w) in enumerate(zip(sets, want))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


# ------------------------------------------------------------------------------------------------ where the rules change over
@pytest.mark.parametrize("B", [248, 249, 256, 257, 264, 265, 1024, 1025])
@pytest.mark.parametrize("ended", [0.0, 0.5])
def test_forks_on_both_sides_of_the_longest_batch_of_one_launch(B, ended):
    """Every warp and every place in the shared tables of children and draws in use, and one row more: launches of their own.  ended: the
    part of the rows that nobody goes on from, whose pages come back and are drawn again in the same call."""
    case = H.pool_case(B, B, 9, 4, 7 * B)
    lens, fixed, held, table, refs, free, taken, rng = case
    some = rng.integers(0, B, B) if ended else np.arange(B)
    parents = np.where(rng.random(B) < 0.6, some, np.arange(B) // 4 * 4)
    parents = np.where(rng.random(B) < ended / 4, -1, parents)
    for most in (5, 20000):
        H.check_fork(H.run_fork(case, parents, 4, most, DEV), C.fork(parents, lens, fixed, held, table, 4, refs, free, taken, most))


def test_a_fork_of_a_long_batch_replayed():
    """The launches of a long batch in a graph, many times over from the same start: the same numbers every time."""
    B, M = 700, 12
    case = H.pool_case(11, B, M, 4, 9000)
    lens, fixed, held, table, refs, free, taken, rng = case
    parents = rng.integers(-1, B, B)
    want = C.fork(parents, lens, fixed, held, table, 4, refs, free, taken, 6000)
    start = [di32(refs), di32(free), di32([taken])]
    state = [x.clone() for x in start]
    new = lambda *s: torch.full(s, -77, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lo, ho, src, dst, counts = new(B, M), new(B), new(B), new(6000), new(6000), new(4)
    ws = torch.full((L.loma_paged_fork_workspace_bytes(B),), 171, dtype=torch.uint8, device=DEV)
    given = [di32(parents), di32(lens), di32(fixed), di32(held), di32(table)]

    def step():
        for x, y in zip(state, start):
            x.copy_(y)
        L.loma_paged_fork(*given, 4, out, lo, ho, *state, src, dst, counts, workspace=ws)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(40):
        for x in (out, lo, ho, src, dst, counts):
            x.fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        H.check_fork((out, lo, ho, *state, (src, dst), counts), want)


@pytest.mark.parametrize("B,M", [(1, 130), (257, 70), (3000, 37), (12000, 5)])
@pytest.mark.parametrize("in_place", [True, False])
def test_release_of_rows_whose_lanes_part(B, M, in_place):
    """Rows that let go of 0, 1, 31, 32, 33 ... pages, so that a warp's lanes go round their loop differently often; several rows to a warp.
    With held_out = held every count is read before it is replaced."""
    n = B * M + 3
    rng = np.random.default_rng(B + M)
    held = rng.integers(0, M + 1, B)
    table = np.where(np.arange(M)[None] < held[:, None], rng.permutation(n)[: B * M].reshape(B, M), -1)
    refs, free, taken = np.zeros(n, dtype=np.int64), np.setdiff1d(np.arange(n), table), 0
    taken = int(held.sum())
    free = np.concatenate([np.full(taken, -1), free])
    case = (held * 4, held * 0, held, table, refs, free, taken, rng)
    gone = rng.choice([0, 1, 31, 32, 33, 64, 65], B)
    keep = np.where(rng.random(B) < 0.2, -1, np.maximum(held - gone, 0) * 4)
    want = C.release(keep, held, table, 4, refs, free, taken)
    for _ in range(3):
        H.check_release(H.run_release(case, keep, 4, DEV, in_place=in_place), want)


@pytest.mark.parametrize("dtype,flags", KINDS)
def test_decode_of_values_near_the_end_of_what_its_sums_carry(dtype, flags):
    """Values of 1e-20: sums over memory are kept times 2^-53, in steps of 2^-96 of an output, of which there are 2^26 to these outputs."""
    s = make(2, 4, 2, 64, [100, 37], [20, 3], 16, dtype)
    for x in ("v", "vt", "vn"):
        s[x] = (s[x] * 1e-20).to(dtype)
    L.loma_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["ps"], di32([0, 0]), di32(s["mems"]))
    call(s, flags)
    check(s, flags)
