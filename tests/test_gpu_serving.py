"""Parity of the serving-step operators with the fp64 oracle: page tables and slot maps (exact), the per-head norm with the
rotary embedding and its gradients, the packed append into cache pages, and decode attention over a shared prefix.

Tolerances.  A bf16 output is off by one rounding, 2^-8 of its value.  In the attention the probabilities are rounded to
bf16 too (2^-8 of each weight at most, so 2^-8 of the weighted mean of |v|).  fp32 work: a dot product of D terms is off by
at most D 2^-24 sum |q_d k_d|, a sum of n terms by n 2^-24 of the sum of their magnitudes; angles are formed in double and
their cos and sin rounded to fp32 (2e-7)."""

import numpy as np
import pytest
import torch

import oracle
from oracle import serving_oracle as S
from paper_2401_09486_b200 import autograd as A
from paper_2401_09486_b200 import binding as L
from paper_2401_09486_b200 import build, synthetic
from tests.test_serving_host import check_extend, exhaust_and_refill, extend_case, huge_extend_case, run_extend

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NOREP = L.LOMA_FLAG_NO_REP_ZONE
U32 = 2.0**-24


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


def half_step(dtype):
    return 2.0**-8 if dtype == torch.bfloat16 else U32


def within(got, want, tol):
    d = np.abs(npf(got) - want)
    assert np.all(np.isfinite(npf(got))) and np.all(d <= tol), (float((d / np.maximum(tol, 1e-300)).max()), float(d.max()))


# ------------------------------------------------------------------------------------------------ page tables
@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("B,M,ps,new_max,n_free,rows", [(1, 1, 1, 1, 1, 1), (5, 4, 4, 9, 30, 40), (37, 6, 16, 50, 40, 601), (3, 0, 8, 4, 2, 9),
                                                        (64, 3, 128, 1, 64, 64), (9, 5, 2, 7, 0, 30), (700, 9, 8, 60, 3000, 20000),
                                                        (5000, 3, 4, 3, 4000, 6000)])
def test_extend_matches_oracle(B, M, ps, new_max, n_free, rows, seed):
    case = extend_case(seed, B, M, ps, new_max, n_free, with_held=seed != 3)
    taken = None if seed < 3 else seed
    got = run_extend(*case[:5], taken, case[5], ps, rows, device=DEV, in_place=seed == 4)
    torch.cuda.synchronize()
    check_extend(got, S.paged_extend(*case[:5], taken, case[5], ps, rows))


def test_extend_one_long_prompt_among_idle_slots_and_unaligned_outputs():
    B, M, ps = 300, 64, 64
    lens, new = np.full(B, -1), np.zeros(B, dtype=np.int64)
    lens[217], new[217] = 100, 3900
    lens[5:9] = 0                                        # requests without new entries
    table = np.where(np.arange(M)[None] < np.where(lens[:, None] > 0, 2, 0), 1000, -1)
    free = np.arange(500)
    want = S.paged_extend(lens, new, None, None, free, None, table, ps, 4001)
    put = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    buf = torch.full((3, 4002), -77, dtype=torch.int32, device=DEV)
    out = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (B + 1, B + 1, B)]
    rows = [buf.view(-1)[i * 4002 + 1:i * 4002 + 4002] for i in range(3)]            # 4-byte aligned only
    tb = put(table)
    L.loma_paged_extend(put(lens), put(new), None, None, put(free), None, tb, ps, *out, *rows)
    torch.cuda.synchronize()
    check_extend([tb, *out, *rows, None], want)
    assert (buf[:, 0] == -77).all()


@pytest.mark.parametrize("in_place", [False, True])       # one launch, and two
def test_extend_saturates(in_place):
    case = huge_extend_case()
    got = run_extend(*case[:5], None, case[5], 4, 50, device=DEV, in_place=in_place)
    torch.cuda.synchronize()
    check_extend(got, S.paged_extend(*case[:5], None, case[5], 4, 50))


def test_extend_replayed_steps_keep_their_state_on_the_device():
    """A captured step that updates held and taken in place hands out every entry once, over replays."""
    B, M, ps = 700, 8, 4
    i32 = dict(dtype=torch.int32, device=DEV)
    lens, held, taken = torch.zeros(B, **i32), torch.zeros(B, **i32), torch.zeros(1, **i32)
    table, free = torch.full((B, M), -1, **i32), torch.randperm(B * M, device=DEV).to(torch.int32)
    rs, pg, sl, sq, po = (torch.empty(n, **i32) for n in (B + 1, B + 1, B, B, B))

    def step():
        L.loma_paged_extend(lens, None, held, None, free, taken, table, ps, rs, pg, held, sl, sq, po)
        lens.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    seen = [sl.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(9):
        graph.replay()
        seen.append(sl.clone())
    torch.cuda.synchronize()
    every = torch.cat(seen)
    assert (every >= 0).all() and every.unique().numel() == 10 * B
    assert int(taken) == 3 * B and (held == 3).all() and torch.equal(free[: 3 * B].sort().values, table[:, :3].flatten().sort().values)


# ------------------------------------------------------------------------------------------------ norm + rotation
LAYOUTS = [(1, 1, 1, 64, 2, 4, 4, 0, 0), (2, 6, 2, 128, 3, 4, 16, 37, 0), (1, 2, 1, 128, 60, 8, 32, 0, 0), (3, 1, 3, 64, 4, 1, 5, 2, 0),
           (1, 4, 4, 128, 0, 4, 0, 1, 0), (2, 2, 2, 128, 3, 8, 32, 100, NOREP), (1, 5, 1, 64, 0, 4, 0, 33, 0)]


def heads(B, H, rows, D, seed, dtype, view):
    if view == "rows_first":                             # a projection's [B, S, H, D] output
        return normal((B, rows, H, D), seed, dtype, 1.5).transpose(1, 2)
    if view == "slice":                                  # rows of a fused [B, S, (H + 1) D] output
        return normal((B, rows, H + 1, D), seed, dtype, 1.5)[:, :, :H].transpose(1, 2)
    return normal((B, H, rows, D), seed, dtype, 1.5)


def empty_like(x):
    """Same shape and strides as x, in storage of its own, filled with a sentinel."""
    span = sum((n - 1) * s for n, s in zip(x.shape, x.stride())) + 1
    return torch.full((span,), 7.0, dtype=x.dtype, device=x.device).as_strided(x.shape, x.stride())


def rope_tol(y, dtype):
    lo, hi = np.split(np.abs(y), 2, -1)
    pair = np.concatenate([lo + hi] * 2, -1)             # either output feature mixes both of the pair
    return half_step(dtype) * np.abs(y) + 4e-6 * pair + 1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("view,ptype", [("plain", 0), ("rows_first", 1), ("slice", 0)])
@pytest.mark.parametrize("B,Hq,Hk,D,n,c,t,tail,flags", LAYOUTS)
def test_norm_rope_forward(B, Hq, Hk, D, n, c, t, tail, flags, view, ptype, dtype):
    rows = oracle.seq_len(n, c, t, tail, flags)
    q, k = heads(B, Hq, rows, D, 1, dtype, view), heads(B, Hk, rows, D, 2, dtype, view)
    wq, wk = 1 + normal((D,), 3, dtype, 0.3), None if view == "slice" else 1 + normal((D,), 4, dtype, 0.3)
    qo, ko = empty_like(q), empty_like(k)
    L.loma_qk_norm_rope_fwd(q, k, wq, wk, qo, ko, n, c, t, tail, flags, eps=1e-5, position_type=ptype)
    torch.cuda.synchronize()
    want = S.qk_norm_rope(npf(q), npf(k), npf(wq), None if wk is None else npf(wk), n, c, t, tail, flags, 1e-5,
                          position_type="contiguous" if ptype else "intermittent")
    for g, w in zip((qo, ko), want):
        within(g, w, rope_tol(w, dtype))
    if view == "slice":                                  # the strided outputs' gaps are left alone
        for b in range(B if rows > 1 else 0):
            gap = qo[b].as_strided((rows - 1, D), (qo.stride(2), 1), qo[b].storage_offset() + Hq * D)
            assert (gap == 7).all()
    q2, k2 = q.clone(), k.clone()                        # in place
    L.loma_qk_norm_rope_fwd(q2, k2, wq, wk, q2, k2, n, c, t, tail, flags, eps=1e-5, position_type=ptype)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


def test_norm_rope_zero_rows_huge_values_and_one_tensor():
    D, rows = 128, 70
    q = normal((1, 2, rows, D), 5)
    q[0, 0, 3] = 0                                       # a row of zeros has a norm of sqrt(eps), not of zero
    q[0, 1, 5] *= 1e15
    q[0, 1, 6] *= 1e-18
    qo, ko = empty_like(q), torch.empty(1, 0, rows, D, device=DEV)
    L.loma_qk_norm_rope_fwd(q, ko, None, None, qo, ko, 0, 4, 0, rows)
    torch.cuda.synchronize()
    want = S.qk_norm_rope(npf(q), npf(q), None, None, 0, 4, 0, rows)[0]
    within(qo, want, rope_tol(want, torch.float32))
    assert (qo[0, 0, 3] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("view", ["plain", "rows_first"])
@pytest.mark.parametrize("B,Hq,Hk,D,n,c,t,tail,flags", [x for x in LAYOUTS if x[4] != 60] + [(2, 40, 8, 64, 1, 2, 3, 1, 0)])
def test_norm_rope_backward(B, Hq, Hk, D, n, c, t, tail, flags, view, dtype):
    rows = oracle.seq_len(n, c, t, tail, flags)
    q, k = heads(B, Hq, rows, D, 1, dtype, view), heads(B, Hk, rows, D, 2, dtype, view)
    gq, gk = heads(B, Hq, rows, D, 3, dtype, view), heads(B, Hk, rows, D, 4, dtype, view)
    wq, wk = (1 + normal((D,), s, dtype, 0.3) for s in (5, 6))
    dq, dk, dwq, dwk = empty_like(q), empty_like(k), torch.empty_like(wq), torch.empty_like(wk)
    ws = torch.full((L.loma_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, D, n, c, t, tail, flags),), 0xFF, dtype=torch.uint8, device=DEV)
    run = lambda *out: L.loma_qk_norm_rope_bwd(q, k, wq, wk, gq, gk, *out, n, c, t, tail, flags, ws, 1e-5)  # noqa: E731
    run(dq, dk, dwq, dwk)
    torch.cuda.synchronize()
    f = [npf(x) for x in (q, k, wq, wk, gq, gk)]
    want = S.qk_norm_rope_bwd(*f, n, c, t, tail, flags, 1e-5)
    for g, w, x, gr, wt in ((dq, want[0], f[0], f[4], f[2]), (dk, want[1], f[1], f[5], f[3])):
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5)
        lo, hi = np.split(np.abs(gr), 2, -1)
        u = np.concatenate([lo + hi] * 2, -1) * np.abs(wt)                      # bounds |w u|
        size = r * (u + np.abs(x) * r * r * (u * np.abs(x)).mean(-1, keepdims=True))
        within(g, w, half_step(dtype) * np.abs(w) + 4e-6 * size + 1e-6)
    for g, w, x, gr in ((dwq, want[2], f[0], f[4]), (dwk, want[3], f[1], f[5])):
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5)
        lo, hi = np.split(np.abs(gr), 2, -1)
        total = (np.concatenate([lo + hi] * 2, -1) * np.abs(x) * r).sum((0, 1, 2))
        within(g, w, half_step(dtype) * np.abs(w) + (B * (Hq + Hk) + 100) * U32 * total + 1e-6)
    first = [x.clone() for x in (dq, dk, dwq, dwk)]
    dq2, dk2, dwq2 = empty_like(q), empty_like(k), torch.empty_like(wq)
    run(dq2, dk2, dwq2, None)                            # bit for bit again, and without one of the gains
    assert all(torch.equal(a, b) for a, b in zip(first, (dq2, dk2, dwq2)))


def test_norm_rope_backward_without_rows_clears_the_gains():
    q, k = torch.empty(1, 2, 0, 64, device=DEV), torch.empty(1, 1, 0, 64, device=DEV)
    dw = torch.full((2, 64), 3.0, device=DEV)
    L.loma_qk_norm_rope_bwd(q, k, None, None, q.clone(), k.clone(), q.clone(), k.clone(), dw[0], dw[1], 0, 4, 0, 0)
    assert (dw == 0).all()


def test_norm_rope_autograd_broadcast_inputs_and_captured_step():
    """Gradients through the autograd op (an expanded k gets the sum over its copies), eager and from a captured graph."""
    B, H, D, n, c, t = 2, 4, 64, 2, 2, 3
    rows = oracle.seq_len(n, c, t)
    q, k1 = normal((B, H, rows, D), 1), normal((B, 1, rows, D), 2)
    wq, wk = 1 + normal((D,), 3, std=0.3), 1 + normal((D,), 4, std=0.3)
    gq, gk = normal((B, H, rows, D), 5), normal((B, H, rows, D), 6)

    def step(*leaves):
        a, b = A.loma_qk_norm_rope(leaves[0], leaves[1].expand(B, H, rows, D), leaves[2], leaves[3], n, c, t)
        return torch.autograd.grad((a * gq).sum() + (b * gk).sum(), leaves)

    leaves = [x.clone().requires_grad_() for x in (q, k1, wq, wk)]
    eager = [x.clone() for x in step(*leaves)]
    f = [npf(x) for x in (q, k1.expand(B, H, rows, D), wq, wk, gq, gk)]
    want = list(S.qk_norm_rope_bwd(*f, n, c, t))
    want[1] = want[1].sum(1, keepdims=True)
    for g, w in zip(eager, want):
        within(g, w, 1e-4 * max(1.0, np.abs(w).max()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*leaves)
    with torch.no_grad():
        leaves[0].mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    fresh = step(*leaves)
    assert all(torch.equal(a, b) for a, b in zip(captured, fresh))
    assert torch.equal(fresh[0], eager[0]) and torch.equal(fresh[2], -eager[2])     # dq is even in q, dwq odd


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Hq,Hk,D,ps", [(1, 1, 1, 64, 1), (7, 6, 2, 128, 16), (33, 32, 8, 128, 64), (200, 3, 3, 64, 12), (5, 40, 40, 128, 8), (9, 0, 2, 64, 4),
                                          (9, 2, 0, 64, 4)])
def test_append(T, Hq, Hk, D, ps, dtype):
    n_pages = T // ps + 3
    qkv = normal((T, (Hq + 2 * Hk) * D), 1, dtype, 1.5)
    q, k, v = (x.unflatten(1, (-1, D)) if x.numel() else x.reshape(T, 0, D) for x in qkv.split([Hq * D, Hk * D, Hk * D], 1))
    wq, wk = 1 + normal((D,), 3, dtype, 0.3), 1 + normal((D,), 4, dtype, 0.3)
    rng = np.random.default_rng(T)
    slots = rng.permutation(n_pages * ps)[:T]
    slots[T // 2:: 3] = [-1, n_pages * ps, -2**31][T % 3]                      # padded rows, and rows past the pool
    pos = rng.integers(0, 200000, T)
    qo = torch.full((T, Hq, D), 7.0, dtype=dtype, device=DEV)
    kp, vp = (torch.full((n_pages, Hk, ps, D), 5.0, dtype=dtype, device=DEV) for _ in range(2))
    want = S.qk_norm_rope_append(npf(q), npf(k), npf(v), npf(wq), npf(wk), npf(kp), npf(vp), slots, pos)
    put = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    L.loma_qk_norm_rope_append(q, k, v, wq, wk, qo, kp, vp, put(slots), put(pos))
    torch.cuda.synchronize()
    within(qo, want[0], rope_tol(want[0], dtype))
    within(kp, want[1], rope_tol(want[1], dtype))
    assert np.array_equal(npf(vp), want[2])
    untouched = want[1] == 5.0
    assert np.array_equal(npf(kp)[untouched], want[1][untouched])


def test_append_into_a_contiguous_cache_and_q_in_place():
    B, Hq, Hk, D, cap = 3, 2, 2, 64, 21                                        # 21 rows a page: not a power of two
    q, k, v = (normal((B, 2, D), s) for s in (1, 2, 3))
    kc, vc = (torch.zeros(B, Hk, cap, D, device=DEV) for _ in range(2))
    lens = torch.tensor([4, 0, 20], dtype=torch.int32, device=DEV)
    slots = (torch.arange(B, device=DEV, dtype=torch.int32) * cap + lens).contiguous()
    want = S.qk_norm_rope_append(npf(q), npf(k), npf(v), None, None, npf(kc), npf(vc), slots.tolist(), lens.tolist())
    L.loma_qk_norm_rope_append(q, k, v, None, None, q, kc, vc, slots, lens)
    torch.cuda.synchronize()
    for g, w in zip((q, kc, vc), want):
        within(g, w, rope_tol(w, torch.float32))


# ------------------------------------------------------------------------------------------------ shared-prefix decode
def shared_case(B, Hq, Hkv, D, P, lens, ps, dtype, seed=0, poison=float("nan"), new=True, extra_cap=3, q_std=1.0):
    """Device tensors of one call (everything a request may not see is `poison`) and the oracle's inputs."""
    mx = max([0, *lens])
    s = {"q": normal((B, Hq, 1, D), seed + 1, dtype, q_std), "kn": normal((B, Hkv, 1, D), seed + 2, dtype), "vn": normal((B, Hkv, 1, D), seed + 3, dtype)}
    kp, vp = normal((Hkv, P, D), seed + 4, dtype), normal((Hkv, P, D), seed + 5, dtype)
    own = [None if n < 0 else tuple(normal((Hkv, n + 1, D), seed + 10 + 2 * b + i, dtype) for i in (0, 1)) for b, n in enumerate(lens)]
    for b, n in enumerate(lens):
        if n >= 0 and new:
            own[b][0][:, n], own[b][1][:, n] = s["kn"][b, :, 0], s["vn"][b, :, 0]
        if n < 0:
            s["q"][b] = poison
    full = lambda *shape: torch.full(shape, poison, dtype=dtype, device=DEV)  # noqa: E731
    if ps == 0:
        s["kp"], s["vp"] = full(Hkv, P + extra_cap, D), full(Hkv, P + extra_cap, D)
        s["kp"][:, :P], s["vp"][:, :P] = kp, vp
        s["kc"], s["vc"] = full(B, Hkv, mx + 1 + extra_cap, D), full(B, Hkv, mx + 1 + extra_cap, D)
        for b, n in enumerate(lens):
            if n >= 0:
                rows = n if new else n + 1
                s["kc"][b, :, :rows], s["vc"][b, :, :rows] = own[b][0][:, :rows], own[b][1][:, :rows]
    else:
        M, Mp = mx // ps + 1, -(-P // ps)
        n_pages = B * M + Mp + 2
        ids = np.random.default_rng(seed).permutation(n_pages)
        table, ptable = ids[: B * M].reshape(B, M), ids[B * M: B * M + Mp]
        s["kc"], s["vc"] = full(n_pages, Hkv, ps, D), full(n_pages, Hkv, ps, D)
        for cache, pre, i in ((s["kc"], kp, 0), (s["vc"], vp, 1)):
            for j in range(Mp):
                m = min(ps, P - j * ps)
                cache[int(ptable[j]), :, :m] = pre[:, j * ps:j * ps + m]
            for b, n in enumerate(lens):
                for j in range(0 if n < 0 else -(-(n if new else n + 1) // ps)):
                    m = min(ps, (n if new else n + 1) - j * ps)
                    cache[int(table[b, j]), :, :m] = own[b][i][:, j * ps:j * ps + m]
        s["table"] = torch.tensor(table, dtype=torch.int32, device=DEV)
        s["ptable"] = torch.tensor(ptable, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["o"], s["lse"] = torch.full((B, Hq, 1, D), 9.0, dtype=dtype, device=DEV), torch.full((B, Hq), 9.0, device=DEV)
    s["ws"] = torch.full((L.loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, P, mx),), 0xFF, dtype=torch.uint8, device=DEV)
    s |= {"P": P, "mx": mx, "ps": ps, "new": new, "own": own, "pre": (kp, vp)}
    return s


def call_shared(s, flags=0, lse=True, **kw):
    kn, vn = (s["kn"], s["vn"]) if s["new"] else (None, None)
    if s["ps"] == 0:
        L.loma_decode_attn_shared(s["q"], kn, vn, s["kp"], s["vp"], s["P"], s["kc"], s["vc"], s["o"], s["lse"] if lse else None, s["lens"], s["mx"],
                                  workspace=s["ws"], flags=flags, **kw)
    else:
        L.loma_decode_attn_shared_paged(s["q"], kn, vn, s["kc"], s["vc"], s["ptable"], s["P"], s["table"], s["o"], s["lse"] if lse else None, s["lens"],
                                        s["mx"], workspace=s["ws"], flags=flags, **kw)


def check_shared(s, scale=None, dtype=None):
    dtype = s["q"].dtype
    q = npf(s["q"])[:, :, 0]
    D = q.shape[-1]
    own = [(None, None) if x is None else (npf(x[0]), npf(x[1])) for x in s["own"]]
    kp, vp = (npf(x) for x in s["pre"])
    live = [b for b, x in enumerate(own) if x[0] is not None]
    o, lse, o_abs = S.decode_attn_shared(np.nan_to_num(q), [x[0] for x in own], [x[1] for x in own], kp, vp, scale)
    g = q.shape[1] // kp.shape[0]
    sc = D**-0.5 if scale is None else scale
    # largest sum |q_d k_d| a score of the sequence's heads can have, bounded through the row norms
    eps_s = np.zeros(lse.shape)
    for b in live:
        kmax = np.sqrt(max((kp**2).sum(-1).max(initial=0), (own[b][0] ** 2).sum(-1).max()))
        eps_s[b] = (D + 4) * U32 * np.sqrt((q[b] ** 2).sum(-1)) * kmax * sc
    keys = s["P"] + s["mx"] + 1
    step = half_step(dtype)
    rel = (step if dtype == torch.bfloat16 else 0) + 2 * eps_s + (keys + 64) * U32 + 1e-6
    got, glse = s["o"][:, :, 0], s["lse"]
    within(got[live], o[live], (step * np.abs(o) + rel[..., None] * o_abs)[live])
    within(glse[live], lse[live], (eps_s + (keys + 64) * U32 + 1e-6 * (1 + np.abs(lse)))[live])
    idle = [b for b in range(len(own)) if b not in live]
    assert (got[idle] == 9.0).all() and (glse[idle] == 9.0).all()


def caches_after(s, before):
    """The caches differ from before by the new tokens' rows only."""
    for cache, old, new in ((s["kc"], before[0], s["kn"]), (s["vc"], before[1], s["vn"])):
        want = old.clone()
        for b, n in enumerate(s["lens"].tolist()):
            if n >= 0 and s["new"]:
                if s["ps"] == 0:
                    want[b, :, n] = new[b, :, 0]
                else:
                    want[int(s["table"][b, n // s["ps"]]), :, n % s["ps"]] = new[b, :, 0]
        assert torch.equal(cache.view(torch.int16 if cache.element_size() == 2 else torch.int32),
                           want.view(torch.int16 if cache.element_size() == 2 else torch.int32))


SHARED = [
    # B, Hq, Hkv, D, P, lens, ps
    (1, 1, 1, 64, 1, [0], 0),
    (1, 1, 1, 128, 0, [0], 0),                                    # no prefix, an empty cache: the new token alone
    (2, 4, 2, 64, 127, [5, -1], 0),
    (3, 3, 1, 128, 128, [0, 64, 130], 0),
    (5, 5, 5, 128, 129, [1, 2, -1, 700, 63], 0),
    (9, 16, 2, 128, 1000, [3, 0, 15, 16, 17, -1, 300, 31, 32], 0),
    (40, 8, 2, 64, 640, [7 * i % 90 - 1 for i in range(40)], 0),  # 160 query rows per kv head: a partial second tile
    (70, 32, 8, 128, 257, [i for i in range(70)], 0),
    (2, 40, 2, 128, 300, [200, 3], 0),                            # groups of 20
    (4, 9, 1, 64, 77, [1, 0, 5, 9], 0),
    (2, 4, 2, 64, 100, [5, 40], 8),
    (3, 8, 8, 128, 500, [0, -1, 131], 16),
    (9, 16, 2, 128, 1030, [3, 0, 15, 16, 17, -1, 300, 31, 32], 64),
    (2, 2, 2, 128, 260, [127, 128], 128),
    (2, 4, 4, 64, 300, [100, 255], 256),
    (3, 4, 2, 128, 45, [6, 1, 9], 1),                             # pages of fewer than 8 rows
    (3, 4, 2, 64, 45, [6, 1, 9], 4),
    (2, 4, 2, 128, 0, [100, 5], 16),
    (1500, 1, 1, 64, 20, [13 * i % 61 - 1 for i in range(1500)], 0),         # several sequences to a group of the own scan
    (9, 16, 8, 128, 100, [2000, 1999, 0, -1, 777, 1500, 16, 15, 2000], 0),   # shares that hold parts of several sequences
    (6, 8, 4, 64, 300, [900, 3, -1, 500, 0, 899], 8),
    (40, 64, 4, 64, 500, [i % 20 for i in range(40)], 16),                   # 640 query rows per kv head, groups of 16
    (3, 40, 2, 128, 200, [100, -1, 3], 0),                                   # groups of 20, short own caches
    (3, 4, 2, 64, 90, [-1, -1, -1], 0),                                      # nothing but idle slots
]
WIDE = (130, 100, 100, 64, 1300, [i % 5 for i in range(130)], 0)             # prefix shares that end inside a kv head, two row tiles


@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared_decode(case, dtype, flags):
    s = shared_case(*SHARED[case], dtype, seed=100 * case)
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s, flags)
    torch.cuda.synchronize()
    check_shared(s)
    caches_after(s, before)
    first = s["o"].clone()
    call_shared(s, flags, lse=False)                              # the appended row is written again: bit for bit the same
    torch.cuda.synchronize()
    assert torch.equal(first, s["o"])


@pytest.mark.parametrize("case", [(1, 1, 1, 64, 100, [0], 0), (1, 1, 1, 128, 1000, [0], 0), (1, 8, 2, 128, 300, [2], 0), (2, 4, 1, 64, 70, [-1, 3], 0),
                                  (1, 2, 2, 64, 333, [4], 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_decode_caches_of_a_few_rows(case, dtype):
    """Own caches around 16 rows in all, below which a tile of them is no tile: prefix and own part take one path together."""
    s = shared_case(*case, dtype, seed=7)
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)
    caches_after(s, before)


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_decode_all_idle_under_a_high_bound(ps, dtype):
    s = shared_case(3, 4, 2, 64, 90, [300, 20, 4], ps, dtype, seed=9)
    s["lens"].fill_(-1)
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s)
    torch.cuda.synchronize()
    assert (s["o"] == 9.0).all() and (s["lse"] == 9.0).all() and L.loma_device_status() == 0
    caches_after(s, before)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_decode_pool_of_one_page(dtype):
    """A pool of 8 rows in all, fewer than a tile has, that holds the sequence's entries and no prefix."""
    s = shared_case(1, 2, 1, 64, 0, [5], 8, dtype, seed=21)
    page = int(s["table"][0, 0])
    s["kc"], s["vc"] = s["kc"][page:page + 1].clone(), s["vc"][page:page + 1].clone()
    s["table"].zero_()
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)
    caches_after(s, before)


@pytest.mark.parametrize("P,ps,D", [(48000, 0, 64), (12000, 16, 64), (12000, 16, 128)])
def test_shared_decode_prefix_cut_for_two_ctas_per_sm(P, ps, D):
    """Prefixes so much longer than the own caches that they are cut twice as finely."""
    s = shared_case(2, 8, 8, D, P, [3, 200], ps, torch.bfloat16, seed=41)
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)


def test_shared_decode_prefix_shares_across_heads():
    s = shared_case(*WIDE, torch.bfloat16, seed=77)
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_decode_replayed_with_new_inputs(ps, dtype):
    """Captured once, replayed with other queries, tokens and lengths (fewer and more than at capture): the eager call's bits."""
    first = shared_case(12, 8, 2, 128, 900, [300, 20, -1, 0] * 3, ps, dtype, seed=31)
    other = shared_case(12, 8, 2, 128, 900, [17, -1, 300, 255] * 3, ps, dtype, seed=32)
    call_shared(other)
    torch.cuda.synchronize()
    want = other["o"].clone(), other["lse"].clone()
    check_shared(other)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call_shared(first)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call_shared(first)
    graph.replay()
    torch.cuda.synchronize()
    check_shared(first)
    for k, v in other.items():
        if isinstance(v, torch.Tensor) and k != "ws":
            first[k].copy_(v)
    first["o"].fill_(9.0), first["lse"].fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first["o"], want[0]) and torch.equal(first["lse"], want[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ps", [0, 16])
def test_shared_decode_token_already_stored_own_scale(ps, dtype):
    s = shared_case(4, 8, 2, 128, 200, [0, 33, -1, 64], ps, dtype, seed=7, new=False)
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s, softmax_scale=0.03)
    torch.cuda.synchronize()
    check_shared(s, scale=0.03)
    caches_after(s, before)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_decode_long_prefix_sharp_scores(dtype):
    """Scores up to about +-40: the maximum moves far along the prefix, and most weights vanish."""
    s = shared_case(6, 8, 2, 128, 5000, [10, 0, 200, 64, 5, 6], 0, dtype, seed=11, q_std=4.0)
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)


def test_shared_decode_lengths_above_the_bound_count_as_the_bound():
    s = shared_case(2, 2, 2, 64, 50, [20, 20], 0, torch.bfloat16, seed=3)
    s["lens"] = torch.tensor([2**31 - 1, 21], dtype=torch.int32, device=DEV)
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)


def test_shared_decode_tables_out_of_range_stay_in_the_pool():
    """Page numbers outside the pool are clamped to it: the call reads and writes nothing else (values are not looked at)."""
    s = shared_case(2, 4, 2, 64, 100, [5, 40], 16, torch.bfloat16, seed=5, poison=1.0)
    s["ptable"][1], s["ptable"][2], s["table"][1, 0] = 2**31 - 1, -5, 10**6
    call_shared(s)
    torch.cuda.synchronize()
    assert torch.isfinite(s["o"].float()).all() and L.loma_device_status() == 0


@pytest.mark.parametrize("ps", [0, 64])
def test_shared_decode_offsets_beyond_32_bits(ps):
    """Own entries that lie more than 2^31 elements into their cache."""
    B, Hkv, D, n = 3, 8, 128, 70
    dtype = torch.bfloat16
    s = shared_case(B, 8, Hkv, D, 40, [n, 5, n], ps, dtype, seed=13)
    if ps == 0:
        cap = 2**31 // (2 * Hkv * D) + 1000                        # sequence 2 starts beyond 2^31 elements
        for name in ("kc", "vc"):
            big = torch.zeros(B, Hkv, cap, D, dtype=dtype, device=DEV)
            big[:, :, : s[name].shape[2]] = s[name]
            s[name] = big
    else:
        far = 2**31 // (Hkv * ps * D) + 5
        for name in ("kc", "vc"):
            big = torch.zeros(far + s[name].shape[0], Hkv, ps, D, dtype=dtype, device=DEV)
            big[far:] = s[name]
            s[name] = big
        s["table"] += far
        s["ptable"] += far
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)


def test_shared_decode_concurrent_streams_and_other_devices_refused():
    cases = [shared_case(20, 8, 2, 128, 700 + 50 * i, [5 * i + j for j in range(20)], 0, torch.bfloat16, seed=200 + i) for i in range(4)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(cases, streams):
            with torch.cuda.stream(st):
                call_shared(s)
    torch.cuda.synchronize()
    for s in cases:
        check_shared(s)
    s = cases[0]
    s["lens"] = s["lens"].cpu()
    with pytest.raises(ValueError):
        call_shared(s)


# ------------------------------------------------------------------------------------------------ one serving step
def test_serving_step_eager_and_captured():
    """Tables and slots, norm + rotation into the pages, attention: three steps of a batch over a shared prefix, the page state
    kept on the device, eager against the oracle and then replayed from one captured graph with the same results."""
    B, Hq, Hkv, D, ps, M, P, steps = 5, 8, 2, 64, 8, 4, 30, 3
    Mp, n_pages, dtype = -(-P // ps), 40, torch.bfloat16
    wq, wk = 1 + normal((D,), 1, dtype, 0.2), 1 + normal((D,), 2, dtype, 0.2)
    inputs = [normal((B, (Hq + 2 * Hkv) * D), 10 + i, dtype) for i in range(steps)]
    i32 = dict(dtype=torch.int32, device=DEV)
    start = torch.tensor([6, 0, -1, 15, 7], **i32)
    pool0 = [normal((n_pages, Hkv, ps, D), 20 + i, dtype) for i in (0, 1)]

    def fresh():
        s = {"lens": start.clone(), "held": (start.clamp(min=0) + ps - 1) // ps, "taken": torch.zeros(1, **i32), "free": torch.arange(25, 40, **i32),
             "table": torch.full((B, M), -1, **i32), "ptable": torch.arange(Mp, **i32), "qkv": inputs[0].clone()}
        s["held"] = s["held"].to(torch.int32)
        for b, n in enumerate(s["held"].tolist()):
            s["table"][b, :n] = torch.arange(10 + 3 * b, 10 + 3 * b + n, **i32)
        s["rs"], s["pg"] = torch.empty(B + 1, **i32), torch.empty(B + 1, **i32)
        s["sl"], s["sq"], s["po"] = (torch.empty(B, **i32) for _ in range(3))
        s["kp"], s["vp"] = pool0[0].clone(), pool0[1].clone()
        s["q"], s["o"] = torch.zeros(B, Hq, D, dtype=dtype, device=DEV), torch.zeros(B, Hq, 1, D, dtype=dtype, device=DEV)
        s["qb"] = torch.zeros(B, Hq, 1, D, dtype=dtype, device=DEV)
        s["ws"] = torch.empty(L.loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, P, M * ps - 1), dtype=torch.uint8, device=DEV)
        return s

    def step(s):
        L.loma_paged_extend(s["lens"], None, s["held"], s["lens"] + P, s["free"], s["taken"], s["table"], ps, s["rs"], s["pg"], s["held"], s["sl"],
                            s["sq"], s["po"])
        rows = s["sq"].clamp(min=0).long()                        # packed rows: the live sequences in order
        x = s["qkv"][rows]
        q, k, v = (y.unflatten(1, (-1, D)) for y in x.split([Hq * D, Hkv * D, Hkv * D], 1))
        L.loma_qk_norm_rope_append(q, k, v, wq, wk, s["q"], s["kp"], s["vp"], s["sl"], s["po"])
        s["qb"].zero_()
        s["qb"].index_copy_(0, torch.where(s["sq"] >= 0, s["sq"].long(), 2), s["q"][:, :, None])    # sequence 2 is idle
        L.loma_decode_attn_shared_paged(s["qb"], None, None, s["kp"], s["vp"], s["ptable"], P, s["table"], s["o"], None, s["lens"], M * ps - 1,
                                        workspace=s["ws"])
        s["lens"].add_((s["lens"] >= 0).to(torch.int32))

    eager = fresh()
    outs = []
    for i in range(steps):
        before = {k: eager[k].clone() for k in ("lens", "held", "taken", "table", "kp", "vp")}
        eager["qkv"].copy_(inputs[i])
        step(eager)
        torch.cuda.synchronize()
        outs.append(eager["o"].clone())
        lens = before["lens"].tolist()
        tab, _, _, held, slots, seq, pos, taken = S.paged_extend(lens, None, before["held"].tolist(), [n + P for n in lens], eager["free"].tolist(),
                                                                 int(before["taken"]), before["table"].cpu().numpy(), ps, B)
        assert np.array_equal(eager["table"].cpu().numpy(), tab) and np.array_equal(eager["held"].cpu().numpy(), held) and int(eager["taken"]) == taken
        x = npf(inputs[i])[np.maximum(seq, 0)].reshape(B, -1, D)
        want_q, want_k, _ = S.qk_norm_rope_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], npf(wq), npf(wk), npf(before["kp"]), npf(before["vp"]),
                                                  slots, pos)
        within(eager["kp"], want_k, rope_tol(want_k, dtype))
        # attention from the stored (rounded) keys and the rounded queries
        kp, vp, qb = npf(eager["kp"]), npf(eager["vp"]), npf(eager["qb"])[:, :, 0]
        pre = [np.concatenate([p[j] for j in range(Mp)], 1)[:, :P] for p in (kp, vp)]
        own = [[None if n < 0 else np.concatenate([p[j] for j in tab[b, : n // ps + 1]], 1)[:, : n + 1] for b, n in enumerate(lens)] for p in (kp, vp)]
        o, _, o_abs = S.decode_attn_shared(qb, own[0], own[1], *pre)
        live = [b for b, n in enumerate(lens) if n >= 0]
        within(eager["o"][live, :, 0], o[live], (2.0**-8 * (np.abs(o) + o_abs) + 1e-4 * o_abs + 1e-6)[live])

    state = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(state)
    for k, v in fresh().items():
        state[k].copy_(v)
    for i in range(steps):
        state["qkv"].copy_(inputs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(state["o"], outs[i])
    for k in ("table", "held", "taken", "kp", "vp", "lens"):
        assert torch.equal(state[k], eager[k])


# ------------------------------------------------------------------------------------------------ short free lists
@pytest.mark.parametrize("B,n_first", [(5, 3), (3000, 700)])
def test_extend_counts_only_the_pages_it_hands_out(B, n_first):
    table, free = exhaust_and_refill(DEV, B=B, n_first=n_first)
    assert torch.equal(table[:, 0], free[:B]) and (table[:, 1:] == -1).all()


# ------------------------------------------------------------------------------------------------ tokens without a page
@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("missing", [-1, -2**31, 10**6])
@pytest.mark.parametrize("mx", [20, 300])                       # sequences that stay whole, and ones that are cut
def test_shared_decode_token_without_a_page_is_not_stored(mx, missing, dtype, flags):
    """The page of sequence 0's new token is not in the pool: the token is attended to, and no page changes for it."""
    s = shared_case(3, 4, 2, 64, 30, [16, 5, mx], 16, dtype, seed=5, poison=0.0)
    s["table"][0, 1] = missing
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s, flags)
    torch.cuda.synchronize()
    check_shared(s)
    s["lens"][0] = -1                                           # nothing stored for it
    caches_after(s, before)


def test_extend_out_of_pages_then_decode_keeps_the_other_requests():
    """A free list that ends one page short, and the token stored by the attention: page 0 belongs to another request."""
    B, Hq, Hkv, D, ps, dtype = 2, 4, 2, 64, 8, torch.bfloat16
    i32 = dict(dtype=torch.int32, device=DEV)
    kp, vp = (normal((3, Hkv, ps, D), s, dtype) for s in (1, 2))
    table, lens = torch.tensor([[0, -1], [1, -1]], **i32), torch.tensor([8, 8], **i32)
    rs, pg, held, sl, sq, po = (torch.empty(n, **i32) for n in (3, 3, 2, 2, 2, 2))
    L.loma_paged_extend(lens, None, None, None, torch.tensor([2], **i32), None, table, ps, rs, pg, held, sl, sq, po)
    assert table.tolist() == [[0, 2], [1, -1]] and sl.tolist() == [16, -1] and int(pg[2]) == 2
    kn, vn = (normal((B, Hkv, 1, D), s, dtype) for s in (3, 4))
    want = [x.clone() for x in (kp, vp)]
    want[0][2, :, 0], want[1][2, :, 0] = kn[0, :, 0], vn[0, :, 0]
    o = torch.empty(B, Hq, 1, D, dtype=dtype, device=DEV)
    ws = torch.empty(L.loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, 0, 15), dtype=torch.uint8, device=DEV)
    L.loma_decode_attn_shared_paged(normal((B, Hq, 1, D), 5, dtype), kn, vn, kp, vp, None, 0, table, o, None, lens, 15, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1]) and torch.isfinite(o.float()).all()


# ------------------------------------------------------------------------------------------------ NaN
@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("where", ["prefix", "own", "token", "query"])
@pytest.mark.parametrize("case", [(1, 4, 2, 64, 20, [5], 0), (2, 4, 2, 128, 40, [300, 200], 0), (3, 8, 2, 128, 3000, [400, 3, 900], 16),
                                  (40, 8, 2, 64, 640, [200] * 40, 0), (128, 8, 8, 64, 300, [170] * 128, 0), (3, 8, 2, 64, 33, [9, -1, 40], 16)])
def test_shared_decode_nan_reaches_the_outputs(case, where, dtype, flags):
    """One NaN key that a row sees makes the row NaN, whichever part of the keys it lies in and however the parts are joined;
    rows that do not see it stay as they were."""
    clean, s = shared_case(*case, dtype, seed=61), shared_case(*case, dtype, seed=61)
    nan = float("nan")
    if where == "prefix":
        (s["kc"][int(s["ptable"][0])] if s["ps"] else s["kp"])[:, 3] = nan
    elif where == "own":
        (s["kc"][int(s["table"][0, 0])] if s["ps"] else s["kc"][0])[:, 1] = nan
    else:
        s["kn" if where == "token" else "q"][0] = nan
    for x in (clean, s):
        call_shared(x, flags)
    torch.cuda.synchronize()
    check_shared(clean)
    live = [b for b, n in enumerate(case[5]) if n >= 0]
    hit = live if where == "prefix" else [0]
    rest = [b for b in range(case[0]) if b not in hit]
    assert torch.isnan(s["o"][hit].float()).all() and torch.isnan(s["lse"][hit]).all()
    assert torch.equal(s["o"][rest], clean["o"][rest]) and torch.equal(s["lse"][rest], clean["lse"][rest])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("n", [20, 200])
def test_shared_decode_a_whole_part_of_nan(n, where, dtype):
    """Every score of one part is NaN, so no maximum of it is a number."""
    s = shared_case(1, 4, 2, 64, 40, [n], 0, dtype, seed=62)
    for x in [s["kp"]] if where == "prefix" else [s["kc"], s["kn"]]:
        x.fill_(float("nan"))
    call_shared(s)
    torch.cuda.synchronize()
    assert torch.isnan(s["o"].float()).all() and torch.isnan(s["lse"]).all()


@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("n", [20, 200])
def test_shared_decode_a_part_without_weight(n, dtype, flags):
    """Prefix scores of -inf: the prefix has no weight."""
    s = shared_case(2, 4, 2, 64, 100, [n, 3], 0, dtype, seed=63)
    s["q"].fill_(1.0)
    s["kp"][:, :100] = 0
    s["kp"][:, :100, 0] = -float("inf")
    s["pre"] = tuple(x[:, :0] for x in s["pre"])                # as if there were none
    call_shared(s, flags)
    torch.cuda.synchronize()
    check_shared(s)


@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("where", ["prefix", "token"])
@pytest.mark.parametrize("P,n,ps,D", [(37, 5, 0, 64), (37, 20, 16, 128), (37, 5, 4, 64), (65, 200, 0, 128), (31, 16, 1, 64)])
def test_shared_decode_infinite_value_at_the_end_of_a_tile(P, n, ps, D, where, dtype, flags):
    """V of the last key of a partial tile is infinite: that feature is infinite, as the mean says, and the others are not NaN."""
    s = shared_case(2, 4, 2, D, P, [n, n], ps, dtype, seed=8)
    inf = float("inf")
    if where == "token":
        s["vn"][:, :, 0, 1] = inf
    elif ps:
        s["vc"][int(s["ptable"][(P - 1) // ps]), :, (P - 1) % ps, 1] = inf
    else:
        s["vp"][:, P - 1, 1] = inf
    call_shared(s, flags)
    torch.cuda.synchronize()
    o = s["o"].float()
    assert (o[..., 1] == inf).all() and torch.isfinite(o[..., 2:]).all() and torch.isfinite(o[..., 0]).all()


# ------------------------------------------------------------------------------------------------ views at any address
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_rope_autograd_takes_views_at_any_address(dtype):
    """Inputs that are contiguous slices of one flat buffer, and outputs joined behind a single number, so that their gradients
    are contiguous slices too: the results of the same call on tensors of their own."""
    D, rows = 64, 7
    shapes = [(1, 2, rows, D), (1, 1, rows, D), (D,), (D,)]
    sizes = [int(np.prod(x)) for x in shapes]
    coef = normal((1 + sum(sizes[:2]),), 9, dtype)

    def run(leaves):
        a, b = A.loma_qk_norm_rope(*leaves, 0, 4, 0, rows)
        joined = torch.cat([torch.zeros(1, dtype=dtype, device=DEV), a.reshape(-1), b.reshape(-1)])
        return [a, b, *torch.autograd.grad((joined * coef).sum(), leaves)]

    flat = normal((1 + sum(sizes),), 1, dtype)
    views, at = [], 1
    for n, shape in zip(sizes, shapes):
        views.append(flat[at:at + n].view(shape).requires_grad_())
        at += n
    assert all(x.data_ptr() % 16 for x in views)
    got, want = run(views), run([x.detach().clone().requires_grad_() for x in views])
    assert all(torch.equal(x, y) for x, y in zip(got, want))
