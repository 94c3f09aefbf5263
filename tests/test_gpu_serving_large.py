"""The serving-step operators and the per-head norm at sizes where their loops run: a lane's fetch ring goes round several times,
a warp crosses from one row to the next, a thread takes a second set of rows, an online softmax moves its reference with
results already behind it, and offsets pass 2^31 elements.  The references are plain fp64 torch operations (gradients by
autograd through them), the NumPy oracle where it is quick enough.

Tolerances as in test_gpu_serving.py: one rounding of the output, 4e-6 of the rotated pair for fp32 work (angles, a norm of at
most 128 features, a few products), and n 2^-24 of the sum of magnitudes for a sum of n terms."""

import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

import oracle
from oracle import serving_oracle as S
from paper_2401_09486_b200 import binding as L
from paper_2401_09486_b200 import build
from tests.test_gpu_serving import DEV, U32, _library, call_shared, caches_after, check_shared, empty_like, half_step, normal, shared_case  # noqa: F401
from tests.test_serving_host import check_extend, extend_case, run_extend

pytestmark = pytest.mark.gpu


def heads(B, H, rows, D, seed, dtype, view):
    """[B, H, rows, D]: plain, a projection's [B, S, H, D] output, or a part of a fused [B, S, (H + 1) D] one."""
    shape = (B, H, rows, D) if view == "plain" else (B, rows, H + (view == "slice"), D)
    x = (1.5 * torch.randn(shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed))).to(dtype)
    return x if view == "plain" else x[:, :, :H].transpose(1, 2)


def rotate(x, pos):
    """Rows x [..., S, D] (fp64) turned by their ids."""
    half = x.shape[-1] // 2
    angle = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / x.shape[-1])
    c, s, lo, hi = angle.cos(), angle.sin(), x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def norm_rope(x, w, pos, eps):
    return rotate(x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * w, pos)


def pair_sum(y):
    lo, hi = y.abs().chunk(2, -1)
    return torch.cat([lo + hi, lo + hi], -1)


def close(got, want, tol):
    d = (got.double() - want).abs()
    assert torch.isfinite(got).all() and bool((d <= tol).all()), (float((d / tol).max()), float(d.max()))


# B, Hq, Hk, D, n, c, t, tail: 20 and more pairs of batch and head to a lane
LONG = [(4, 32, 8, 128, 16, 4, 16, 5), (3, 20, 20, 64, 0, 4, 0, 3001), (1, 64, 32, 128, 24, 8, 16, 0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("view", ["plain", "rows_first", "slice"])
@pytest.mark.parametrize("B,Hq,Hk,D,n,c,t,tail", LONG)
def test_norm_rope_walks_many_pairs(B, Hq, Hk, D, n, c, t, tail, view, dtype):
    rows, eps = oracle.seq_len(n, c, t, tail), 1e-5
    q, k = heads(B, Hq, rows, D, 1, dtype, view), heads(B, Hk, rows, D, 2, dtype, view)
    gq, gk = heads(B, Hq, rows, D, 3, dtype, view), heads(B, Hk, rows, D, 4, dtype, view)
    wq, wk = (1 + normal((D,), s, dtype, 0.3) for s in (5, 6))
    pos = torch.tensor(oracle.position_ids(n, c, t, tail), dtype=torch.float64, device=DEV)
    qo, ko, dq, dk, dwq, dwk = (empty_like(x) for x in (q, k, q, k, wq, wk))
    ws = torch.full((L.loma_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, D, n, c, t, tail),), 0xFF, dtype=torch.uint8, device=DEV)
    L.loma_qk_norm_rope_fwd(q, k, wq, wk, qo, ko, n, c, t, tail, eps=eps)
    L.loma_qk_norm_rope_bwd(q, k, wq, wk, gq, gk, dq, dk, dwq, dwk, n, c, t, tail, 0, ws, eps)
    torch.cuda.synchronize()
    for x, w, g, y, dx, dw in ((q, wq, gq, qo, dq, dwq), (k, wk, gk, ko, dk, dwk)):
        x, w, g = x.double().requires_grad_(), w.double().requires_grad_(), g.double()
        want = norm_rope(x, w, pos, eps)
        want_dx, want_dw = torch.autograd.grad((want * g).sum(), (x, w))
        with torch.no_grad():
            close(y, want, half_step(dtype) * want.abs() + 4e-6 * pair_sum(want) + 1e-6)
            r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
            u = pair_sum(g)                                        # bounds the gradient before the rotation
            size = r * (u * w.abs() + x.abs() * r.square() * (u * w.abs() * x.abs()).mean(-1, keepdim=True))
            close(dx, want_dx, half_step(dtype) * want_dx.abs() + 4e-6 * size + 1e-6)
            total = (u * x.abs() * r).sum((0, 1, 2))
            close(dw, want_dw, half_step(dtype) * want_dw.abs() + (B * (Hq + Hk) + 100) * U32 * total + 1e-6)
    q2, k2 = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
    if q2.stride() == q.stride() and k2.stride() == k.stride():
        L.loma_qk_norm_rope_fwd(q2, k2, wq, wk, q2, k2, n, c, t, tail, eps=eps)            # in place
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
    first = [x.clone() for x in (dq, dk, dwq, dwk)]
    L.loma_qk_norm_rope_bwd(q, k, wq, wk, gq, gk, dq, dk, dwq, dwk, n, c, t, tail, 0, ws, eps)
    assert all(torch.equal(a, b) for a, b in zip(first, (dq, dk, dwq, dwk)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Hq,Hk,D,ps", [(500, 32, 8, 128, 16), (1500, 12, 4, 64, 64), (8000, 32, 8, 128, 64), (3600, 3, 3, 64, 12), (20001, 1, 1, 128, 8)])
def test_append_many_rows(T, Hq, Hk, D, ps, dtype):
    """Several steps to a row and, beyond 3552 rows, several rows to a warp; every fifth row has no slot."""
    n_pages = T // ps + 3
    qkv = normal((T, (Hq + 2 * Hk) * D), 1, dtype, 1.5)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hk * D, Hk * D], 1))
    wq, wk = 1 + normal((D,), 3, dtype, 0.3), 1 + normal((D,), 4, dtype, 0.3)
    rng = np.random.default_rng(T)
    slots = torch.tensor(rng.permutation(n_pages * ps)[:T], dtype=torch.int32, device=DEV)
    slots[::5] = -1
    pos = torch.tensor(rng.integers(0, 200000, T), dtype=torch.int32, device=DEV)
    qo = torch.full((T, Hq, D), 7.0, dtype=dtype, device=DEV)
    kp, vp = (torch.full((n_pages, Hk, ps, D), 5.0, dtype=dtype, device=DEV) for _ in range(2))
    L.loma_qk_norm_rope_append(q, k, v, wq, wk, qo, kp, vp, slots, pos)
    torch.cuda.synchronize()
    want_q, want_k = (norm_rope(x.double().transpose(0, 1), w.double(), pos.double(), 1e-6).transpose(0, 1) for x, w in ((q, wq), (k, wk)))
    tol = lambda y: half_step(dtype) * y.abs() + 4e-6 * pair_sum(y) + 1e-6  # noqa: E731
    close(qo, want_q, tol(want_q))
    stored = slots >= 0
    page, row = (slots[stored] // ps).long(), (slots[stored] % ps).long()
    close(kp[page, :, row], want_k[stored], tol(want_k[stored]))
    assert torch.equal(vp[page, :, row], v[stored])
    kp[page, :, row], vp[page, :, row] = 5.0, 5.0
    assert (kp == 5.0).all() and (vp == 5.0).all()                 # nothing else was written


@pytest.mark.parametrize("in_place", [False, True])               # one launch, and two
@pytest.mark.parametrize("extra", [1, 200000])
def test_extend_more_rows_than_one_round(in_place, extra):
    """Some 770000 rows: threads take a second set of rows, the last of them behind the packed batch."""
    case = extend_case(4 if in_place else 2, 1400, 20, 64, 1100, 30000)
    total = int(np.where(case[0] < 0, 0, np.maximum(case[1], 0)).sum())
    assert total > 296 * 512 * 4
    taken = 5 if in_place else None
    got = run_extend(*case[:5], taken, case[5], 64, total + extra, device=DEV, in_place=in_place)
    torch.cuda.synchronize()
    check_extend(got, S.paged_extend(*case[:5], taken, case[5], 64, total + extra))


def ramp_scores(s, prefix, own):
    """Feature 0 adds the key's ramp times the query's factor to the score (in natural units).  Factors differ from row to row, so
    that rows side by side move their references at different keys or not at all."""
    B, Hq, _, D = s["q"].shape
    factor = torch.tensor([1.0, 0.5, -1.0, 0.0, 0.75], device=DEV)[torch.arange(B * Hq, device=DEV) % 5].view(B, Hq, 1)
    s["q"][..., 0] = (factor * D**0.5).to(s["q"].dtype)            # times the scale of D^-1/2: the key's feature is the score
    kp = s["pre"][0]
    kp[..., 0] = prefix(kp.shape[1]).to(kp.dtype)
    s["kp"][:, : s["P"]] = kp
    for b, n in enumerate(s["lens"].tolist()):
        if n >= 0:
            k = s["own"][b][0]
            k[..., 0] = own(n + 1).to(k.dtype)
            s["kc"][b, :, :n], s["kn"][b, :, 0] = k[:, :n], k[:, n]


RAMPS = {
    "slow": lambda n: 0.0125 * torch.arange(n, device=DEV),                    # a move of the reference every ten or so blocks
    "steep": lambda n: 0.05 * torch.arange(n, device=DEV) - 20.0,              # one every other block
    "jump": lambda n: torch.where(torch.arange(n, device=DEV) % 701 == 700, 0.03 * torch.arange(n, device=DEV), 0.0),
}


@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, L.LOMA_FLAG_FORCE_GENERIC)])
@pytest.mark.parametrize("shape", [(4, 16, 8, 128, 12000, [3000, 2999, -1, 3100], 0),      # ten blocks to a prefix and to an own worker
                                   (70, 16, 4, 64, 6000, [20 + 9 * i for i in range(70)], 0),   # three tiles of query rows
                                   (3, 32, 2, 128, 40000, [100, 0, 900], 0)])                   # sixteen heads to a kv head
@pytest.mark.parametrize("ramp", list(RAMPS))
def test_shared_decode_reference_moves_over_a_worker(ramp, shape, dtype, flags):
    """Scores that grow along the keys, so that outputs and sums collected under an old reference are rescaled again and again
    within one worker's stay in a sequence."""
    s = shared_case(*shape, dtype, seed=91)
    ramp_scores(s, RAMPS[ramp], RAMPS[ramp])
    call_shared(s, flags)
    torch.cuda.synchronize()
    check_shared(s)


# ------------------------------------------------------------------------------------------------ offsets beyond 2^31 elements
@pytest.mark.parametrize("ps", [0, 64])
def test_shared_decode_on_cuda_cores_offsets_beyond_32_bits(ps):
    B, Hkv, D, n, dtype = 3, 8, 128, 70, torch.bfloat16
    s = shared_case(B, 8, Hkv, D, 40, [n, 5, n], ps, dtype, seed=13)
    lead = 2**31 // (2 * Hkv * D) + 1000 if ps == 0 else 2**31 // (Hkv * ps * D) + 5
    for name in ("kc", "vc"):
        big = torch.zeros(*((B, Hkv, lead, D) if ps == 0 else (lead + s[name].shape[0], Hkv, ps, D)), dtype=dtype, device=DEV)
        if ps == 0:
            big[:, :, : s[name].shape[2]] = s[name]
        else:
            big[lead:] = s[name]
        s[name] = big
    if ps:
        s["table"] += lead
        s["ptable"] += lead
    call_shared(s, L.LOMA_FLAG_FORCE_GENERIC)
    torch.cuda.synchronize()
    check_shared(s)
    b = 2                                                          # the new token's row, beyond 2^31 elements as well
    for cache, new in ((s["kc"], s["kn"]), (s["vc"], s["vn"])):
        row = cache[b, :, n] if ps == 0 else cache[int(s["table"][b, n // ps]), :, n % ps]
        assert torch.equal(row, new[b, :, 0])


def test_append_offsets_beyond_32_bits():
    Hk, D, ps, dtype = 4, 128, 64, torch.bfloat16
    far = 2**31 // (Hk * ps * D) + 3
    kp, vp = (torch.zeros(far + 1, Hk, ps, D, dtype=dtype, device=DEV) for _ in range(2))
    q, k, v = normal((2, 2, D), 1, dtype), normal((2, Hk, D), 2, dtype), normal((2, Hk, D), 3, dtype)
    slots, pos = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([far * ps + 63, 1], [100000, 7]))
    L.loma_qk_norm_rope_append(q, k, v, None, None, torch.empty_like(q), kp, vp, slots, pos)
    torch.cuda.synchronize()
    want = norm_rope(k.double().transpose(0, 1), 1.0, pos.double(), 1e-6).transpose(0, 1)
    tol = half_step(dtype) * want.abs() + 4e-6 * pair_sum(want) + 1e-6
    for i, (page, row) in enumerate(((far, 63), (0, 1))):
        close(kp[page, :, row], want[i], tol[i])
        assert torch.equal(vp[page, :, row], v[i])
    for pool in (kp, vp):
        pool[far, :, 63], pool[0, :, 1] = 0, 0
        assert not pool.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16])
def test_norm_rope_strides_beyond_32_bits(dtype):
    """Batch elements 2^31 elements apart, heads and rows far apart within them."""
    B, H, rows, D, eps = 2, 3, 5, 64, 1e-6
    strides = (2**31 + 64 * 8, 2**29, 2**26, 1)
    span = sum((m - 1) * st for m, st in zip((B, H, rows, D), strides)) + 1
    q, g, dq, out = (torch.zeros(span, dtype=dtype, device=DEV).as_strided((B, H, rows, D), strides) for _ in range(4))
    q.copy_(normal((B, H, rows, D), 1, dtype, 1.5))
    g.copy_(normal((B, H, rows, D), 2, dtype))
    k = torch.empty(B, 0, rows, D, dtype=dtype, device=DEV)
    ws = torch.empty(L.loma_qk_norm_rope_bwd_workspace_bytes(B, H, 0, D, 0, 4, 0, rows), dtype=torch.uint8, device=DEV)
    L.loma_qk_norm_rope_fwd(q, k, None, None, out, k, 0, 4, 0, rows)
    L.loma_qk_norm_rope_bwd(q, k, None, None, g, k, dq, k.clone(), None, None, 0, 4, 0, rows, 0, ws)
    torch.cuda.synchronize()
    x = q.double().requires_grad_()
    want = norm_rope(x, 1.0, torch.arange(rows, dtype=torch.float64, device=DEV), eps)
    want_dx, = torch.autograd.grad((want * g.double()).sum(), x)
    with torch.no_grad():
        close(out, want, half_step(dtype) * want.abs() + 4e-6 * pair_sum(want) + 1e-6)
        r, u = (x.square().mean(-1, keepdim=True) + eps).rsqrt(), pair_sum(g.double())
        size = r * (u + x.abs() * r.square() * (u * x.abs()).mean(-1, keepdim=True))
        close(dq, want_dx, half_step(dtype) * want_dx.abs() + 4e-6 * size + 1e-6)


def test_extend_table_beyond_32_bits():
    """Block tables of 2^30 columns: the third sequence's row of the table starts at entry 2^31."""
    M = 2**30
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.zeros(3, M, **i32)
    table[2, M - 5:] = torch.tensor([11, 12, 13, -1, -1], **i32)
    lens, new, held = (torch.tensor(x, **i32) for x in ([0, -1, M - 3], [2, 5, 4], [1, 0, M - 2]))
    table[0, 0] = 9
    for in_place in (False, True):
        rs, pg, sl, sq, po = (torch.full((m,), -77, **i32) for m in (4, 4, 8, 8, 8))
        h = held.clone()
        tab = table if in_place else table.clone()
        L.loma_paged_extend(lens, new, h, None, torch.tensor([20, 21, 22], **i32), None, tab, 1, rs, pg, h if in_place else torch.empty_like(h), sl, sq, po)
        torch.cuda.synchronize()
        assert rs.tolist() == [0, 2, 2, 6] and pg.tolist() == [0, 1, 1, 3]
        assert sl.tolist() == [9, 20, 13, 21, 22, -1, -1, -1] and sq.tolist() == [0, 0, 2, 2, 2, 2, -1, -1]
        assert po.tolist() == [0, 1, M - 3, M - 2, M - 1, M, 0, 0]
        assert tab[0, :3].tolist() == [9, 20, 0] and tab[2, M - 6:].tolist() == [0, 11, 12, 13, 21, 22] and not tab[1].any() and not tab[2, : M - 5].any()
        del tab


# ------------------------------------------------------------------------------------------------ how calls meet
@pytest.mark.parametrize("ps", [0, 8, 16])
def test_shared_decode_two_sequences_to_a_warp(ps):
    """Short own caches of more (sequence, kv head) pairs than there are warps: each stays whole, and a warp takes two."""
    s = shared_case(70, 16, 16, 128, 100, [(7 * i) % 100 - 1 for i in range(70)], ps, torch.bfloat16, seed=4)
    before = s["kc"].clone(), s["vc"].clone()
    call_shared(s)
    torch.cuda.synchronize()
    check_shared(s)
    caches_after(s, before)


def test_shared_decode_from_several_threads():
    cases = [shared_case(4 + i, 8, 2, 128, 300 + i, [10 * j for j in range(4 + i)], 0, torch.bfloat16, seed=300 + i) for i in range(6)]
    torch.cuda.synchronize()

    def work(s):
        torch.cuda.set_device(0)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(100):
                call_shared(s)
        stream.synchronize()

    with ThreadPoolExecutor(len(cases)) as pool:
        list(pool.map(work, cases))
    for s in cases:
        check_shared(s)


def test_a_step_run_again_after_the_list_ran_short():
    """A step that ran out of pages is run again with a longer list: the outputs of a step that had enough from the start."""
    B, Hq, Hkv, D, ps, M, P, dtype = 6, 8, 2, 64, 8, 3, 20, torch.bfloat16
    i32 = dict(dtype=torch.int32, device=DEV)
    lens, w = torch.tensor([8, 5, 16, 0, 15, 8], **i32), 1 + normal((D,), 1, dtype, 0.2)
    qkv, pools = normal((B, Hq + 2 * Hkv, D), 2, dtype), [normal((40, Hkv, ps, D), s, dtype) for s in (3, 4)]
    ptable, free = torch.arange(3, **i32), torch.arange(30, 40, **i32)

    def run(list_lengths):
        held, taken, table = ((lens + ps - 1) // ps).to(torch.int32), torch.zeros(1, **i32), torch.full((B, M), -1, **i32)
        for b, n in enumerate(held.tolist()):
            table[b, :n] = torch.arange(4 + 3 * b, 4 + 3 * b + n, **i32)
        kp, vp = (x.clone() for x in pools)
        rs, pg, sl, sq, po = (torch.empty(n, **i32) for n in (B + 1, B + 1, B, B, B))
        q, o = torch.empty(B, Hq, D, dtype=dtype, device=DEV), torch.empty(B, Hq, 1, D, dtype=dtype, device=DEV)
        ws = torch.empty(L.loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, P, M * ps - 1), dtype=torch.uint8, device=DEV)
        for n in list_lengths:
            L.loma_paged_extend(lens, None, held, lens + P, free[:n], taken, table, ps, rs, pg, held, sl, sq, po)
            L.loma_qk_norm_rope_append(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], w, w, q, kp, vp, sl, po)
            L.loma_decode_attn_shared_paged(q[:, :, None], None, None, kp, vp, ptable, P, table, o, None, lens, M * ps - 1, workspace=ws)
            short = int(pg[-1]) > n
        assert not short and (sl >= 0).all() and int(taken) == 4
        return o, kp

    (enough, _), (again, kp) = run([10]), run([2, 10])
    assert torch.equal(enough, again)
    assert torch.equal(kp[:4], pools[0][:4])                      # the prefix's pages and one nobody has


FIRST_CALL = """
import sys
import torch
from paper_2401_09486_b200 import binding as L
d, bf, which = "cuda:0", torch.bfloat16, sys.argv[1]
i = lambda *x: torch.tensor(x, dtype=torch.int32, device=d)
n32 = lambda *x: torch.zeros(*x, dtype=torch.int32, device=d)
q, kn, kp = torch.randn(2, 4, 1, 64, device=d).to(bf), torch.randn(2, 2, 1, 64, device=d).to(bf), torch.randn(2, 100, 64, device=d).to(bf)
kc, vc, o = torch.zeros(2, 2, 64, 64, device=d, dtype=bf), torch.zeros(2, 2, 64, 64, device=d, dtype=bf), torch.zeros_like(q)
x, y, z, dw = torch.randn(2, 4, 10, 64, device=d), torch.zeros(2, 4, 10, 64, device=d), torch.zeros(2, 4, 10, 64, device=d), torch.zeros(64, device=d)
lens, table, sl, qo = i(3, 40), torch.full((2, 4), -1, dtype=torch.int32, device=d), n32(2), torch.zeros(2, 4, 64, device=d, dtype=bf)
ws = torch.zeros(max(L.loma_decode_shared_workspace_bytes(2, 4, 2, 64, 100, 63), 1 << 20), dtype=torch.uint8, device=d)
calls = {"shared": (o, lambda: L.loma_decode_attn_shared(q, kn, kn, kp, kp, 100, kc, vc, o, None, lens, 63, workspace=ws)),
         "extend": (sl, lambda: L.loma_paged_extend(lens, None, None, None, i9, n32(1), table, 16, n32(3), n32(3), n32(2), sl, n32(2), n32(2))),
         "norm": (y, lambda: L.loma_qk_norm_rope_fwd(x, x, None, None, y, z, 0, 4, 0, 10)),
         "backward": (dw, lambda: L.loma_qk_norm_rope_bwd(x, x, None, None, x + 1, x, y, z, dw, None, 0, 4, 0, 10, 0, ws)),
         "append": (qo, lambda: L.loma_qk_norm_rope_append(q[:, :, 0], kn[:, :, 0], kn[:, :, 0], None, None, qo, kc, vc, lens, lens))}
i9 = torch.arange(5, 14, dtype=torch.int32, device=d)
out, call = calls[which]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
graph.replay()
torch.cuda.synchronize()
assert out.ne(0).any()
print("captured")
"""


@pytest.mark.parametrize("which", ["shared", "extend", "norm", "backward", "append"])
def test_the_first_call_of_a_process_may_be_captured(which):
    out = subprocess.run([sys.executable, "-c", FIRST_CALL, which], capture_output=True, text=True, timeout=300, cwd=build.ROOT)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]
