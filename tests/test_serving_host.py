"""Host-side checks of the serving-step entry points that need no GPU: refusals before any CUDA call, and the host form of
loma_paged_extend against the oracle."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2401_09486_b200 import binding as L
from paper_2401_09486_b200 import build

INVALID, UNSUPPORTED, ALIGNMENT, CAPACITY, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return L.lib()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32)


def run_extend(cache_lens, new_lens, held, pos0, free, taken, table, ps, rows, device="cpu", in_place=False):
    B = len(cache_lens)
    put = lambda x: None if x is None else i32(x).to(device)  # noqa: E731
    a = [put(x) for x in (cache_lens, new_lens, held, pos0, free)]
    tk, tb = None if taken is None else i32([taken]).to(device), i32(table).to(device).reshape(B, -1)
    out = [torch.full((n,), -77, dtype=torch.int32, device=device) for n in (B + 1, B + 1, B, rows, rows, rows)]
    if in_place:
        out[2] = a[2]
    L.loma_paged_extend(*a, tk, tb, ps, *out)
    return [tb, *out, tk]


def check_extend(got, want):
    for g, w in zip(got[:-1], want[:-1]):
        assert np.array_equal(g.cpu().numpy().astype(np.int64), w), (g, w)
    if got[-1] is not None:
        assert int(got[-1]) == want[-1]


def extend_case(seed, B, M, ps, new_max, n_free, with_held=True):
    rng = np.random.default_rng(seed)
    lens = rng.integers(-1, M * ps + 2, B) if seed % 2 else rng.integers(0, max(1, M * ps // 2), B)
    new = rng.integers(-1, new_max + 1, B)
    held = np.clip(-(-np.maximum(lens, 0) // ps) + rng.integers(0, 2, B), 0, M) if with_held else None
    have = held if with_held else np.minimum(-(-np.maximum(lens, 0) // ps), M)
    ids = rng.permutation(n_free + B * M)
    table = np.where(np.arange(M)[None] < have[:, None], ids[n_free:].reshape(B, M), -1)
    return lens, new, held, rng.integers(0, 1000, B), ids[:n_free], table


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("B,M,ps,new_max,n_free,rows", [(1, 1, 1, 1, 1, 1), (5, 4, 4, 9, 30, 40), (37, 6, 16, 50, 40, 600), (3, 0, 8, 4, 2, 9),
                                                        (64, 3, 128, 1, 64, 64), (9, 5, 2, 7, 0, 30)])
def test_host_extend_matches_oracle(lib, seed, B, M, ps, new_max, n_free, rows):
    case = extend_case(seed, B, M, ps, new_max, n_free, with_held=seed != 3)
    taken = None if seed < 3 else seed
    got = run_extend(*case[:5], taken, case[5], ps, rows, in_place=seed == 4)
    check_extend(got, S.paged_extend(*case[:5], taken, case[5], ps, rows))


def test_host_extend_defaults_and_steps_in_place(lib):
    """new_lens, held and pos0 left out; then a run of single-token steps that keep held and taken in place."""
    lens, table, free = [3, 4, -1], [[8, -1], [2, -1], [-1, -1]], [11, 12, 13]
    check_extend(run_extend(lens, None, None, None, free, None, table, 4, 3), S.paged_extend(lens, None, None, None, free, None, table, 4, 3))
    B, M, ps = 3, 4, 2
    held, taken, table = torch.zeros(B, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.full((B, M), -1, dtype=torch.int32)
    free = torch.arange(100, 112, dtype=torch.int32)
    lens = torch.tensor([0, 2, 5], dtype=torch.int32)
    rs, pg = torch.empty(B + 1, dtype=torch.int32), torch.empty(B + 1, dtype=torch.int32)
    sl, sq, po = (torch.empty(B, dtype=torch.int32) for _ in range(3))
    seen = set()
    for _ in range(3):
        L.loma_paged_extend(lens, None, held, None, free, taken, table, ps, rs, pg, held, sl, sq, po)
        live = [int(x) for x in sl if x >= 0]
        assert not seen & set(live) and len(set(live)) == len(live)       # no entry is handed out twice
        seen |= set(live)
        lens += 1
    assert int(taken) == int((table >= 0).sum()) and held.tolist() == [2, 3, 4]


def huge_extend_case():
    """Sums and positions far beyond 32 bits, entries beyond the table, page numbers whose slots do not fit."""
    big = 2**31 - 1
    lens, new = [5, big, 0, -2**31, 3], [big, big, -2**31, big, 4]
    table = [[7, -1, -1], [1, 2, 3], [-1, -1, -1], [9, 9, 9], [big, 4, -1]]
    return lens, new, [1, 3, 0, big, 2], [10, big, 0, 0, big - 1], [40, 41], table


def test_host_extend_saturates(lib):
    case = huge_extend_case()
    got = run_extend(*case[:5], None, case[5], 4, 50)
    check_extend(got, S.paged_extend(*case[:5], None, case[5], 4, 50))
    assert got[1].tolist() == [0] + [2**31 - 1] * 5          # row_start


def test_extend_refusals(lib):
    def call(B=2, ps=4, M=3, rows=4, n_free=2, dev=0, swap=None):
        p = {n: 0x10000 + 0x1000 * i for i, n in enumerate("lens new held pos free taken table rs pg ho sl sq po".split())}
        p |= swap or {}
        return lib.loma_paged_extend(B, ps, M, rows, n_free, *p.values(), dev, None)

    assert call(B=-1, dev=1) == INVALID and call(ps=3, dev=1) == INVALID and call(ps=0, dev=1) == INVALID and call(ps=1 << 17, dev=1) == INVALID
    assert call(M=1 << 30, dev=1) == INVALID and call(rows=-1, dev=1) == INVALID and call(n_free=-1, dev=1) == INVALID
    for name in ("lens", "table", "rs", "pg", "ho", "sl", "sq", "po", "free"):
        assert call(dev=1, swap={name: None}) == INVALID, name
        assert call(dev=1, swap={name: 0x10002}) == ALIGNMENT, name
    for name in ("ho", "sl", "rs", "table", "taken"):
        assert call(dev=1, swap={name: 0x10004}) == INVALID, name           # inside cache_lens
    assert call(dev=1, swap={"sl": 0x20000, "sq": 0x20008}) == INVALID       # two outputs meet
    assert call(dev=1, swap={"ho": 0x12004}) == INVALID                      # shifted against held
    rs = torch.full((1,), 5, dtype=torch.int32)
    pg = torch.full((1,), 5, dtype=torch.int32)
    sl, sq, po = (torch.full((2,), 5, dtype=torch.int32) for _ in range(3))
    e = torch.empty(0, dtype=torch.int32)
    L.loma_paged_extend(e, None, None, None, None, None, e.view(0, 3), 4, rs, pg, e.clone(), sl, sq, po)      # no sequences
    assert rs.tolist() == [0] and pg.tolist() == [0] and sl.tolist() == [-1, -1] and sq.tolist() == [-1, -1] and po.tolist() == [0, 0]
    with pytest.raises(ValueError):
        L.loma_paged_extend(i32([1, 2]), None, None, None, None, None, i32([[1], [2]]), 4, rs, pg, i32([0, 0]), sl, sq, po)   # row_start too short
    with pytest.raises(ValueError):
        L.loma_paged_extend(torch.tensor([1, 2]), None, None, None, None, None, i32([[1], [2]]), 4, i32([0, 0, 0]), i32([0, 0, 0]), i32([0, 0]), sl, sq, po)


def _st(*x):
    return (ctypes.c_int64 * len(x))(*x)


def test_norm_refusals(lib):
    def fwd(q=0x1000, k=0x2000, wq=None, wk=None, qo=0x3000, ko=0x4000, B=1, Hq=2, Hk=1, D=64, n=1, c=2, t=2, tc=4, tail=0, qs=(1280, 640, 64),
            ks=(640, 640, 64), dt=1, pt=0, flags=0):
        return lib.loma_qk_norm_rope_fwd(q, k, wq, wk, qo, ko, B, Hq, Hk, D, n, c, t, tc, tail, qs and _st(*qs), ks and _st(*ks), dt, 0.0, 0.0, pt,
                                         flags, None)

    assert fwd(D=96) == UNSUPPORTED and fwd(dt=7) == UNSUPPORTED and fwd(B=-1) == INVALID and fwd(tc=5) == INVALID
    assert fwd(q=None) == INVALID and fwd(ko=None) == INVALID and fwd(qs=None) == INVALID and fwd(pt=2) == INVALID
    assert fwd(q=0x1008) == ALIGNMENT and fwd(wk=0x1004) == ALIGNMENT and fwd(ks=(0, 0, 68)) == ALIGNMENT
    assert fwd(qs=(1280, 64, 64)) == INVALID and fwd(qs=(1280, 0, 64)) == INVALID and fwd(qs=(1280, 640, 32)) == INVALID
    assert fwd(B=2, qs=(640, 640, 64), ks=(640, 0, 64)) == INVALID           # batch elements on the same rows
    assert fwd(qo=0x4000) == INVALID and fwd(qo=0x2000) == INVALID and fwd(Hq=70000, B=1) == INVALID
    assert fwd(n=0, tail=0) == 0 and fwd(B=0) == 0 and fwd(Hq=0, Hk=0) == 0

    def bwd(outs=(0x7000, 0x8000, 0x9000, 0xa000), ws=0x10000, wsb=1 << 30, n=1, gq=0x5000):
        return lib.loma_qk_norm_rope_bwd(0x1000, 0x2000, 0x3000, 0x4000, gq, 0x6000, *outs, 1, 2, 1, 64, n, 2, 2, 4, 0, _st(1280, 640, 64),
                                         _st(640, 640, 64), 1, 0.0, 0.0, 0, 0, ws, wsb, None)

    need = L.loma_qk_norm_rope_bwd_workspace_bytes(1, 2, 1, 64, 1, 2, 2)
    assert need > 0 and bwd(ws=None) == WORKSPACE and bwd(wsb=need - 1) == WORKSPACE and bwd(ws=0x10010) == ALIGNMENT
    assert bwd(outs=(None, 0x8000, None, None)) == INVALID and bwd(gq=None) == INVALID
    assert bwd(outs=(0x1000, 0x8000, None, None)) == INVALID and bwd(outs=(0x7000, 0x7000, None, None)) == INVALID
    assert bwd(outs=(0x7000, 0x8000, 0x9000, 0x9000)) == INVALID
    assert bwd(outs=(None, None, None, None), n=0) == 0
    assert L.loma_qk_norm_rope_bwd_workspace_bytes(1, 2, 1, 96, 1, 2, 2) == 0


def test_append_refusals(lib):
    def call(q=0x1000, k=0x2000, v=0x3000, qo=0x4000, kp=0x5000, vp=0x6000, sl=0x7000, pos=0x8000, T=2, Hq=2, Hk=1, D=64, ps=5, n=2, qs=(128, 64),
             ks=(64, 64), vs=(64, 64), dt=1, w=None):
        return lib.loma_qk_norm_rope_append(q, k, v, w, None, qo, kp, vp, sl, pos, T, Hq, Hk, D, ps, n, _st(*qs), _st(*ks), _st(*vs), dt, 0.0, 0.0,
                                            None)

    assert call(D=32) == UNSUPPORTED and call(dt=2) == UNSUPPORTED and call(T=-1) == INVALID and call(ps=0) == INVALID and call(n=0) == INVALID
    for name in ("q", "k", "v", "qo", "kp", "vp", "sl", "pos"):
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: 0x9002}) == ALIGNMENT, name
    assert call(qs=(64, 64)) == INVALID and call(ks=(0, 64)) == INVALID and call(vs=(68, 64)) == ALIGNMENT
    assert call(qo=0x1000, qs=(192, 64)) == INVALID and call(kp=0x6000) == INVALID and call(qo=0x5000) == INVALID and call(w=0x1001) == ALIGNMENT
    assert call(T=0) == 0


def test_shared_decode_refusals(lib):
    def call(q=0x1000, kn=0x2000, vn=0x3000, kp=0x4000, vp=0x5000, kc=0x6000, vc=0x7000, o=0x8000, lse=None, B=2, Hq=4, Hkv=2, D=64, pcap=10, plen=9,
             cap=8, lens=0x9000, mx=7, dt=1, flags=0, ws=0x10000, wsb=1 << 40):
        return lib.loma_decode_attn_shared(q, kn, vn, kp, vp, kc, vc, o, lse, B, Hq, Hkv, D, pcap, plen, cap, lens, mx, dt, 0.0, flags, ws, wsb, None)

    assert call(Hq=5) == INVALID and call(Hkv=0) == INVALID and call(D=80) == UNSUPPORTED and call(dt=3) == UNSUPPORTED and call(plen=-1) == INVALID
    assert call(plen=11) == CAPACITY and call(mx=8) == CAPACITY and call(vn=None) == INVALID and call(mx=-1) == INVALID
    for name in ("q", "kc", "vc", "o", "lens", "kp", "vp"):
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: 0x9002}) == ALIGNMENT, name
    need = L.loma_decode_shared_workspace_bytes(2, 4, 2, 64, 9, 7)
    assert need > 0 and call(ws=None) == WORKSPACE and call(wsb=need - 1) == WORKSPACE and call(ws=0x10008) == ALIGNMENT
    assert call(B=0) == 0 and call(B=1 << 22) == INVALID and call(Hq=70000 * 2, Hkv=70000, B=1) == INVALID

    def paged(ps=4, pp=3, plen=9, M=2, n=5, pt=0xa000, bt=0xb000, mx=7, kn=0x2000, ws=0x10000):
        return lib.loma_decode_attn_shared_paged(0x1000, kn, 0x3000, 0x4000, 0x5000, pt, bt, 0x8000, None, 2, 4, 2, 64, ps, pp, plen, M, n, 0x9000, mx,
                                                 1, 0.0, 0, ws, 1 << 40, None)

    assert paged(ps=6) == INVALID and paged(plen=13) == CAPACITY and paged(mx=8) == CAPACITY and paged(pt=None) == INVALID and paged(bt=None) == INVALID
    assert paged(n=0) == INVALID and paged(kn=None) == INVALID and paged(pt=0xa002) == ALIGNMENT and paged(ws=None) == WORKSPACE
    assert L.loma_decode_shared_workspace_bytes(2, 5, 2, 64, 9, 7) == 0 and L.loma_decode_shared_workspace_bytes(0, 4, 2, 64, 9, 7) == 0


def test_shared_workspace_covers_every_size(lib):
    """Never smaller for a longer cache bound or prefix than the partial results of one range need."""
    for B, Hq, Hkv, D, P, mx in ((1, 1, 1, 64, 0, 0), (1, 8, 1, 128, 1, 0), (200, 32, 8, 128, 30000, 4000), (3, 40, 2, 64, 129, 100000)):
        rows = B * Hq * (D + 1) * 4
        assert L.loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, P, mx) >= rows * (1 + (P > 0))


def test_binding_refuses_mismatched_tensors():
    q, k = torch.zeros(1, 2, 10, 64), torch.zeros(1, 1, 10, 64)
    with pytest.raises(ValueError):
        L.loma_qk_norm_rope_fwd(q, k, None, None, torch.zeros(1, 2, 9, 64), k.clone(), 1, 2, 2)
    with pytest.raises(ValueError):
        L.loma_qk_norm_rope_fwd(q, k, torch.zeros(63), None, q.clone(), k.clone(), 1, 2, 2)
    with pytest.raises(ValueError):
        L.loma_qk_norm_rope_fwd(q, k, None, None, q.clone(), k.clone(), 1, 2, 2, 1)       # the layout has 11 rows
    with pytest.raises(ValueError):
        L.loma_qk_norm_rope_append(torch.zeros(3, 2, 64), torch.zeros(3, 1, 64), torch.zeros(3, 1, 64), None, None, torch.zeros(3, 2, 64),
                                   torch.zeros(2, 1, 4, 64), torch.zeros(2, 1, 4, 64), i32([0, 1]), i32([0, 1, 2]))
    with pytest.raises(ValueError):
        L.loma_decode_attn_shared(torch.zeros(2, 2, 1, 64), None, None, torch.zeros(1, 5, 64), torch.zeros(1, 5, 64), 5, torch.zeros(2, 1, 4, 64),
                                  torch.zeros(2, 1, 5, 64), torch.zeros(2, 2, 1, 64), None, i32([0, 0]), 3)


def exhaust_and_refill(device, B=5, ps=2, n_first=3):
    """Steps of one token each over a list that runs short, is tried again twice and then grows: every page goes to one
    sequence, none is passed over.  Returns the table and the pages held."""
    t = dict(dtype=torch.int32, device=device)
    lens, held, taken, table = torch.zeros(B, **t), torch.zeros(B, **t), torch.zeros(1, **t), torch.full((B, 4), -1, **t)
    free = torch.arange(40, 40 + 2 * B, **t)
    rs, pg, sl, sq, po = (torch.empty(n, **t) for n in (B + 1, B + 1, B, B, B))
    for n in (n_first, n_first, n_first, n_first + 1, 2 * B, 2 * B):
        before, had = int(taken), held.clone()
        L.loma_paged_extend(lens, None, held, None, free[:n], taken, table, ps, rs, pg, held, sl, sq, po)
        drawn = int((held - had).sum())
        assert int(taken) == before + drawn <= n                             # what was handed out, no more
        assert int(pg[-1]) == before + int((had == 0).sum())                 # what was asked for: the shortage can be read
    assert int(taken) == B and held.tolist() == [1] * B
    return table, free


def test_host_extend_counts_only_the_pages_it_hands_out(lib):
    table, free = exhaust_and_refill("cpu")
    assert table[:, 0].tolist() == free[:5].tolist() and (table[:, 1:] == -1).all()


def test_host_extend_list_shorter_than_what_was_taken(lib):
    """A list that has been cut below the count keeps the count; the oracle agrees."""
    case = ([0, 3], None, [0, 1], None, [5, 6], 4, [[-1, -1], [9, -1]])
    got = run_extend(*case[:6], case[6], 2, 2)
    check_extend(got, S.paged_extend(*case[:6], case[6], 2, 2))
    assert int(got[-1]) == 4 and got[3].tolist() == [0, 1]


def test_shared_workspace_grows_with_the_sizes(lib):
    """A buffer made for the largest batch, prefix and cache bound serves every smaller call, across the bounds at which the
    cut of a call changes."""
    need = L.loma_decode_shared_workspace_bytes
    assert need(32, 32, 8, 128, 2048, 128) >= need(32, 32, 8, 128, 2048, 127) and need(16, 32, 8, 128, 32768, 8000) >= need(16, 32, 8, 128, 32768, 100)
    assert need(32, 32, 8, 128, 2400, 127) >= need(32, 32, 8, 128, 2304, 127)
    lens = [0, 1, 15, 16, 100, 111, 112, 127, 128, 129, 300, 1500, 8000, 100000]
    prefixes = [0, 1, 31, 32, 33, 64, 65, 200, 1000, 2304, 2400, 4096, 9000, 32768, 200000]
    batches = [1, 2, 3, 5, 8, 16, 31, 32, 33, 37, 64, 65, 128, 200, 300, 1000]
    for Hq, Hkv in ((1, 1), (8, 8), (32, 8), (64, 8), (40, 2), (100, 100), (9, 1)):
        grid = np.array([[[need(B, Hq, Hkv, 64, P, n) for n in lens] for P in prefixes] for B in batches], dtype=np.int64)
        assert all((np.diff(grid, axis=i) >= 0).all() for i in range(3)), (Hq, Hkv)


def test_shared_plan_replayed(lib, tmp_path):
    """Every cut of a shared-prefix call, replayed on the host: blocks and partial results (tests/c_abi/shared_plan_check.cu)."""
    exe = str(tmp_path / "shared_plan_check")
    root, libdir = build.ROOT, build.PKG_DIR
    subprocess.run([build._nvcc(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.INCLUDE, "-I", build.CSRC,
                    os.path.join(root, "tests", "c_abi", "shared_plan_check.cu"), "-o", exe, "-L", libdir, "-lloma", "-Xlinker", f"-rpath={libdir}"],
                   check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and "shared plans ok" in out.stdout, out.stdout + out.stderr


def test_norm_workspace_grows_with_the_sizes(lib):
    """A buffer made for the longest layout and the largest batch serves every smaller call; a few sums of D numbers per CTA."""
    need = L.loma_qk_norm_rope_bwd_workspace_bytes
    rows, batches, heads = [1, 2, 7, 8, 9, *range(20, 9000, 61), 34816, 100000], [1, 2, 3, 4, 9, 64], [(1, 0), (1, 1), (2, 2), (5, 2), (8, 8), (32, 8), (32, 32)]
    for D in (64, 128):
        grid = np.array([[[need(B, hq, hk, D, 0, 4, 0, S) for S in rows] for B in batches] for hq, hk in heads], dtype=np.int64)
        assert all((np.diff(grid, axis=i) >= 0).all() for i in range(3))
        assert grid.max() <= 2 * D * 4 * (100000 // 8 + 1) + 256


def test_build_keeps_the_library_without_the_extension(lib, monkeypatch, tmp_path):
    """A C user's build does not depend on torch's headers or on g++: the library is there, and a warning says what is not."""
    monkeypatch.setattr(build, "MARSHAL_PATH", str(tmp_path / "_marshal.so"))

    def fails(cmd, what, verbose):
        raise RuntimeError(f"{what} failed")

    monkeypatch.setattr(build, "_run", fails)
    with pytest.warns(UserWarning, match="g\\+\\+ failed"):
        assert build.build_library() == build.LIB_PATH
    monkeypatch.setattr(build, "marshal_key", lambda: __import__("no_such_torch"))
    with pytest.warns(UserWarning, match="no_such_torch"):
        assert build.build_library() == build.LIB_PATH


def test_extension_is_built_again_for_another_torch(lib, monkeypatch):
    assert not build._marshal_stale() and L._native().built_for == build.marshal_key()
    monkeypatch.setattr(torch, "__version__", "2.99.0")
    assert build._marshal_stale()
    monkeypatch.setattr(L, "_marshal", None)
    with pytest.raises(RuntimeError, match="was built for"):
        L._native()
