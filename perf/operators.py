"""Cases for the serving-step operators: page tables, per-head norm + rotation, shared-prefix decode attention.

Each case names its operator in "op":

  extend   block tables and slot maps from request lengths (loma_paged_extend)
  norm     RMS norm of every head of q and k with the rotary embedding, training layout (loma_qk_norm_rope_fwd)
  normbwd  its gradients (loma_qk_norm_rope_bwd)
  append   the same for packed new tokens, keys and values written to cache pages (loma_qk_norm_rope_append)
  shared   one new token per sequence over a prefix that the whole batch shares and the sequence's own cache
           (loma_decode_attn_shared, loma_decode_attn_shared_paged)

Where `own` is false, run() computes the operators in elementary torch operations in 32 bits (64 for angles).
"""

import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one generated token for each of 64 running requests, 16-entry pages: what a generation step does first
        {"name": "extend_decode_64", "op": "extend", "B": 64, "ps": 16, "M": 512, "len": 8000, "new": 1},
        # a burst of new prompts of up to 2000 tokens over 64-entry pages, some slots idle
        {"name": "extend_prompts_1000", "op": "extend", "B": 1000, "ps": 64, "M": 128, "len": 500, "new": 2000},
        # the 4608-token training layout, 32 heads
        {"name": "norm_bf16_4608", "op": "norm", "B": 4, "Hq": 32, "Hk": 32, "D": 128, "n": 32, "c": 4, "t": 16, "tail": 0, "dt": "bf16",
         "rows_first": False},
        # a small odd layout with an unfinished chunk, fp32, heads of 64
        {"name": "norm_fp32_small", "op": "norm", "B": 2, "Hq": 6, "Hk": 2, "D": 64, "n": 3, "c": 4, "t": 16, "tail": 37, "dt": "fp32",
         "rows_first": True},
        # gradients for the same layout with grouped heads, q and k as views of a projection's [B, S, H, D] output
        {"name": "normbwd_bf16_4608", "op": "normbwd", "B": 4, "Hq": 32, "Hk": 8, "D": 128, "n": 32, "c": 4, "t": 16, "tail": 0, "dt": "bf16",
         "rows_first": True},
        {"name": "normbwd_fp32_odd", "op": "normbwd", "B": 1, "Hq": 5, "Hk": 5, "D": 64, "n": 7, "c": 3, "t": 7, "tail": 20, "dt": "fp32",
         "rows_first": False},
        # one token for each of 32 requests
        {"name": "append_decode_32", "op": "append", "T": 32, "Hq": 32, "Hk": 8, "D": 128, "ps": 64, "dt": "bf16"},
        # prompt pieces of several requests, 6000 rows together
        {"name": "append_prompts_6000", "op": "append", "T": 6000, "Hq": 32, "Hk": 8, "D": 128, "ps": 64, "dt": "bf16"},
        # few requests over a short shared prompt: latency
        {"name": "shared_small", "op": "shared", "B": 8, "Hq": 8, "Hk": 8, "D": 64, "P": 1000, "len": 64, "ps": 0, "dt": "bf16"},
        # 32 requests, 8192 shared compressed entries, tails of up to 64, 64-entry pages, one head per kv head
        {"name": "shared_paged_8192", "op": "shared", "B": 32, "Hq": 32, "Hk": 32, "D": 128, "P": 8192, "len": 64, "ps": 64, "dt": "bf16"},
        # many requests with grouped heads and long answers of their own
        {"name": "shared_grouped_128", "op": "shared", "B": 128, "Hq": 32, "Hk": 8, "D": 128, "P": 16384, "len": 1500, "ps": 0, "dt": "bf16"},
        # the fp32 path
        {"name": "shared_fp32", "op": "shared", "B": 12, "Hq": 16, "Hk": 4, "D": 128, "P": 2500, "len": 300, "ps": 16, "dt": "fp32"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _cost(c))
    while True:
        op = rng.choice(("extend", "norm", "normbwd", "append", "shared", "shared"))
        D = rng.choice((64, 128))
        dt = rng.choice(("bf16", "bf16", "fp32"))
        Hk = rng.choice((1, 2, 3, 4, 8, 8, 16, 32))
        g = rng.choice((1, 1, 2, 4, 5, 8))
        if op == "extend":
            ps = rng.choice((1, 8, 16, 64, 128))
            c = {"op": op, "B": _log(rng, 1, 4096), "ps": ps, "M": _log(rng, 2, 1024), "len": _log(rng, 1, 8000), "new": _log(rng, 1, 4000)}
        elif op in ("norm", "normbwd"):
            t, r = rng.randint(1, 32), rng.randint(1, 8)
            c = {"op": op, "B": rng.randint(1, 6), "Hq": Hk * g, "Hk": Hk, "D": D, "n": _log(rng, 1, 64), "c": r, "t": t,
                 "tail": rng.randint(0, t * r), "dt": dt, "rows_first": rng.random() < 0.5}
        elif op == "append":
            c = {"op": op, "T": _log(rng, 1, 8000), "Hq": Hk * g, "Hk": Hk, "D": D, "ps": rng.choice((1, 8, 16, 64, 128)), "dt": dt}
        else:
            c = {"op": op, "B": _log(rng, 1, 256), "Hq": Hk * g, "Hk": Hk, "D": D, "P": _log(rng, 1, 30000), "len": _log(rng, 1, 4000),
                 "ps": rng.choice((0, 0, 16, 64, 128)), "dt": dt}
        if _cost(c) <= most[op] and (dt == "bf16" or op != "shared" or work(c)["flops"] <= 2e10):
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _layout_rows(c):
    return c["n"] * c["t"] * (2 * c["c"] + 1) + c["tail"]


def work(case):
    c = case
    es = 2 if c.get("dt") == "bf16" else 4
    if c["op"] == "extend":
        rows = c["B"] if c["new"] == 1 else c["B"] * (c["new"] + 1) / 2 * 0.9
        pages = rows / c["ps"]
        # lengths, new lengths, held pages, first positions; sums, held pages; row outputs; fresh pages read and written
        return {"bytes": 4.0 * (4 * c["B"] + 3 * c["B"] + 3 * rows + 2 * pages), "flops": 0.0}
    if c["op"] in ("norm", "normbwd"):
        e = c["B"] * _layout_rows(c) * (c["Hq"] + c["Hk"]) * c["D"]
        passes = 2 if c["op"] == "norm" else 3
        return {"bytes": float(passes * e * es), "flops": float((8 if passes == 2 else 20) * e)}
    if c["op"] == "append":
        e = c["T"] * (c["Hq"] + 2 * c["Hk"]) * c["D"]
        return {"bytes": float(2 * e * es + 8 * c["T"]), "flops": float(8 * e)}
    mean = c["len"] / 2
    rows = c["B"] * c["Hq"] * c["D"]
    kv = 2.0 * c["Hk"] * c["D"] * (c["P"] + c["B"] * (mean + 2))
    return {"bytes": float(es * (kv + 2 * rows)), "flops": float(4 * rows * (c["P"] + mean + 1))}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, dt, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dt)


def _ints(gen, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=gen, device=DEV, dtype=torch.int32)


def _pages(gen, n):
    return torch.randperm(n, generator=gen, device=DEV).to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = {"c": c}
    if c["op"] == "extend":
        B, ps, M = c["B"], c["ps"], c["M"]
        room = M * ps
        lens = _ints(gen, 0, min(c["len"], room), B)
        new = torch.ones(B, dtype=torch.int32, device=DEV) if c["new"] == 1 else _ints(gen, 0, c["new"], B)
        if c["new"] > 1:  # a slot in ten holds no request
            lens = torch.where(torch.rand(B, generator=gen, device=DEV) < 0.1, -1, lens).to(torch.int32)
        held = (lens.clamp(min=0) + ps - 1) // ps
        held = torch.minimum(held + _ints(gen, 0, 1, B), torch.full_like(held, M)).to(torch.int32)  # pages kept after a compress step
        n_free = max(1, int(c["B"] * (c["new"] + ps) / ps))
        ids = _pages(gen, n_free + B * M)
        table = torch.where(torch.arange(M, device=DEV)[None] < held[:, None], ids[n_free:].view(B, M), -1).to(torch.int32)
        s |= {"lens": lens, "new": new, "held": held, "pos0": lens.clamp(min=0) * 3, "free": ids[:n_free].contiguous(), "table": table.contiguous()}
        rows = B if c["new"] == 1 else max(1, int(B * (c["new"] + 1) * 0.55))
        for name, n in (("row_start", B + 1), ("page_start", B + 1), ("held_out", B), ("slots", rows), ("row_seq", rows), ("row_pos", rows)):
            s[name] = torch.empty(n, dtype=torch.int32, device=DEV)
        return s
    dt, D = DT[c["dt"]], c["D"]
    if c["op"] in ("norm", "normbwd"):
        S = _layout_rows(c)

        def heads(H):
            if c["rows_first"]:
                return _normal(gen, (c["B"], S, H, D), dt, 1.7).transpose(1, 2)
            return _normal(gen, (c["B"], H, S, D), dt, 1.7)

        s |= {"q": heads(c["Hq"]), "k": heads(c["Hk"])}
        s |= {"wq": (1 + _normal(gen, (D,), torch.float32, 0.2)).to(dt), "wk": (1 + _normal(gen, (D,), torch.float32, 0.2)).to(dt)}
        s |= {"q_out": torch.empty_like(s["q"]), "k_out": torch.empty_like(s["k"])}  # outputs, or dq and dk
        if c["op"] == "normbwd":
            s |= {"gq": heads(c["Hq"]), "gk": heads(c["Hk"]), "dwq": torch.empty_like(s["wq"]), "dwk": torch.empty_like(s["wk"])}
            if own:
                from paper_2401_09486_b200 import binding as L

                s["ws"] = torch.empty(max(256, L.loma_qk_norm_rope_bwd_workspace_bytes(c["B"], c["Hq"], c["Hk"], D, c["n"], c["c"], c["t"], c["tail"])),
                                      dtype=torch.uint8, device=DEV)
        return s
    if c["op"] == "append":
        T, ps, Hk = c["T"], c["ps"], c["Hk"]
        n_pages = (T + ps - 1) // ps + 3
        qkv = _normal(gen, (T, (c["Hq"] + 2 * Hk) * D), dt, 1.7)  # one projection's output; the operator takes views of it
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([c["Hq"] * D, Hk * D, Hk * D], 1))
        slots = torch.randperm(n_pages * ps, generator=gen, device=DEV)[:T].to(torch.int32)
        if T > 20:
            slots[-(T // 20):] = -1  # rows of padding behind the last request
        s |= {"q": q, "k": k, "v": v, "slots": slots, "positions": _ints(gen, 0, 100000, T)}
        s |= {"wq": (1 + _normal(gen, (D,), torch.float32, 0.2)).to(dt), "wk": (1 + _normal(gen, (D,), torch.float32, 0.2)).to(dt)}
        s |= {"q_out": torch.empty(T, c["Hq"], D, dtype=dt, device=DEV), "k_pool": torch.zeros(n_pages, Hk, ps, D, dtype=dt, device=DEV),
              "v_pool": torch.zeros(n_pages, Hk, ps, D, dtype=dt, device=DEV)}
        return s
    B, Hk, P, ps = c["B"], c["Hk"], c["P"], c["ps"]
    s |= {"q": _normal(gen, (B, c["Hq"], 1, D), dt), "k_new": _normal(gen, (B, Hk, 1, D), dt), "v_new": _normal(gen, (B, Hk, 1, D), dt)}
    lens = _ints(gen, 0, c["len"], B)
    if B > 6:
        lens[-(B // 6):][::2] = -1  # slots of the batch that hold no request
    s |= {"lens": lens, "o": torch.zeros(B, c["Hq"], 1, D, dtype=dt, device=DEV), "lse": torch.zeros(B, c["Hq"], dtype=torch.float32, device=DEV)}
    if ps == 0:
        cap = c["len"] + 1
        s |= {"kp": _normal(gen, (Hk, P + 5, D), dt), "vp": _normal(gen, (Hk, P + 5, D), dt)}
        s |= {"k_cache": _normal(gen, (B, Hk, cap, D), dt), "v_cache": _normal(gen, (B, Hk, cap, D), dt)}
    else:
        M, Mp = c["len"] // ps + 1, (P + ps - 1) // ps
        n_pages = B * M + Mp
        ids = _pages(gen, n_pages)
        s |= {"k_cache": _normal(gen, (n_pages, Hk, ps, D), dt), "v_cache": _normal(gen, (n_pages, Hk, ps, D), dt)}
        s |= {"table": ids[: B * M].view(B, M).contiguous(), "prefix_table": ids[B * M:].contiguous()}
    if own:
        from paper_2401_09486_b200 import binding as L

        s["ws"] = torch.empty(max(256, L.loma_decode_shared_workspace_bytes(B, c["Hq"], Hk, D, P, c["len"])), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"extend": _extend, "norm": _norm, "normbwd": _normbwd, "append": _append, "shared": _shared}[state["c"]["op"]](state)


def _run_own(s):
    from paper_2401_09486_b200 import binding as L

    c = s["c"]
    if c["op"] == "extend":
        L.loma_paged_extend(s["lens"], s["new"], s["held"], s["pos0"], s["free"], None, s["table"], c["ps"], s["row_start"], s["page_start"],
                            s["held_out"], s["slots"], s["row_seq"], s["row_pos"])
        return [s[k] for k in ("table", "row_start", "page_start", "held_out", "slots", "row_seq", "row_pos")]
    if c["op"] == "norm":
        L.loma_qk_norm_rope_fwd(s["q"], s["k"], s["wq"], s["wk"], s["q_out"], s["k_out"], c["n"], c["c"], c["t"], c["tail"], eps=EPS,
                                theta_base=BASE)
        return s["q_out"], s["k_out"]
    if c["op"] == "normbwd":
        L.loma_qk_norm_rope_bwd(s["q"], s["k"], s["wq"], s["wk"], s["gq"], s["gk"], s["q_out"], s["k_out"], s["dwq"], s["dwk"], c["n"], c["c"],
                                c["t"], c["tail"], workspace=s["ws"], eps=EPS, theta_base=BASE)
        return s["q_out"], s["k_out"], s["dwq"], s["dwk"]
    if c["op"] == "append":
        L.loma_qk_norm_rope_append(s["q"], s["k"], s["v"], s["wq"], s["wk"], s["q_out"], s["k_pool"], s["v_pool"], s["slots"], s["positions"],
                                   eps=EPS, theta_base=BASE)
        return s["q_out"], s["k_pool"], s["v_pool"]
    if c["ps"] == 0:
        L.loma_decode_attn_shared(s["q"], s["k_new"], s["v_new"], s["kp"], s["vp"], c["P"], s["k_cache"], s["v_cache"], s["o"], s["lse"],
                                  s["lens"], c["len"], workspace=s["ws"])
    else:
        L.loma_decode_attn_shared_paged(s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["prefix_table"], c["P"], s["table"],
                                        s["o"], s["lse"], s["lens"], c["len"], workspace=s["ws"])
    return s["o"], s["lse"], s["k_cache"], s["v_cache"]


def _extend(s):
    ps, (B, M), rows, n_free = s["c"]["ps"], s["table"].shape, s["slots"].numel(), s["free"].numel()
    room = M * ps
    lens, held = s["lens"].long().clamp(0, room), s["held"].long().clamp(0, M)
    n = torch.where(s["lens"] < 0, 0, s["new"].long().clamp(min=0))
    fresh = torch.where(n > 0, (((lens + n).clamp(max=room) + ps - 1) // ps - held).clamp(min=0), 0)
    zero = torch.zeros(1, dtype=torch.long, device=n.device)
    row_start, page_start = torch.cat([zero, n.cumsum(0)]), torch.cat([zero, fresh.cumsum(0)])
    got = torch.minimum((n_free - page_start[:-1]).clamp(min=0), fresh)
    col = torch.arange(M, device=n.device)[None]
    at = page_start[:-1, None] + col - held[:, None]
    page = torch.where(at < n_free, s["free"][at.clamp(0, n_free - 1)], -1)
    table = torch.where((col >= held[:, None]) & (col < (held + fresh)[:, None]), page, s["table"])
    r = torch.arange(rows, device=n.device)
    seq = torch.searchsorted(row_start[1:], r, right=True)
    there, b = seq < B, seq.clamp(max=B - 1)
    i = r - row_start[b]
    e = lens[b] + i
    p = table[b, (e // ps).clamp(max=M - 1)].long()
    slots = torch.where(there & (e < room) & (p >= 0), p * ps + e % ps, -1)
    pos = torch.where(there, s["pos0"].long()[b] + i, 0)
    i32 = [x.to(torch.int32) for x in (table, row_start, page_start, held + got, slots, torch.where(there, seq, -1), pos)]
    return i32


def _positions(c):
    """Position ids of the training layout's rows: reading and repetition rows carry their token's, memory row j y*tc + (j+1)c - 1."""
    t, r = c["t"], c["c"]
    tc, span = t * r, t * (2 * r + 1)
    i = torch.arange(_layout_rows(c), device=DEV)
    y, o = i // span, i % span
    whole = torch.where(o < tc, o, torch.where(o < tc + t, (o - tc + 1) * r - 1, o - tc - t)) + y * tc
    return torch.where(i < c["n"] * span, whole, i - c["n"] * span + c["n"] * tc)


def _angles(pos, D):
    a = pos.double()[:, None] * torch.pow(BASE, -2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    return torch.cos(a).float(), torch.sin(a).float()


def _turn(x, cos, sin):
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _normed(x, w, cos, sin):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _turn(x * r * w.float(), cos, sin)


def _norm(s):
    cos, sin = _angles(_positions(s["c"]), s["c"]["D"])
    return tuple(_normed(s[x], s["w" + x], cos, sin).to(s[x].dtype) for x in "qk")


def _normbwd(s):
    cos, sin = _angles(_positions(s["c"]), s["c"]["D"])
    dx, dw = [], []
    for name in "qk":
        x, w, u = s[name].float(), s["w" + name].float(), _turn(s["g" + name].float(), cos, -sin)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        dw.append((u * x * r).sum((0, 1, 2)).to(s[name].dtype))
        dx.append((r * (w * u - x * r * r * (w * u * x).mean(-1, keepdim=True))).to(s[name].dtype))
    return (*dx, *dw)


def _append(s):
    c = s["c"]
    cos, sin = _angles(s["positions"], c["D"])
    cos, sin = cos[:, None], sin[:, None]
    q_out = _normed(s["q"], s["wq"], cos, sin).to(s["q"].dtype)
    k = _normed(s["k"], s["wk"], cos, sin).to(s["q"].dtype)
    # rows without a slot go to one more row behind the pool, which is dropped
    slot = s["slots"].long()
    real = slot >= 0
    for pool, new in ((s["k_pool"], k), (s["v_pool"], s["v"])):
        flat = torch.where(real, slot, pool.shape[0] * c["ps"])
        padded = torch.cat([pool.transpose(1, 2).flatten(0, 1), pool.new_zeros(1, *new.shape[1:])])
        padded[flat] = new
        pool.copy_(padded[:-1].unflatten(0, (-1, c["ps"])).transpose(1, 2))
    return q_out, s["k_pool"], s["v_pool"]


def _own_rows(s):
    """Each sequence's own cache as [B, Hk, rows, D] after the new token went in."""
    c = s["c"]
    b = torch.arange(c["B"], device=DEV)
    slot = s["lens"].long().clamp(min=0)
    idle = (s["lens"] < 0)[:, None, None]
    kc, vc = s["k_cache"], s["v_cache"]
    for cache, new in ((kc, s["k_new"]), (vc, s["v_new"])):
        if c["ps"] == 0:
            cache[b, :, slot] = torch.where(idle, cache[b, :, slot], new[:, :, 0])
        else:
            page, row = s["table"][b, slot // c["ps"]].long(), slot % c["ps"]
            cache[page, :, row] = torch.where(idle, cache[page, :, row], new[:, :, 0])
    if c["ps"] == 0:
        return kc.float(), vc.float()
    return tuple(x[s["table"].long()].transpose(1, 2).flatten(2, 3).float() for x in (kc, vc))


def _shared(s):
    c = s["c"]
    B, Hk, D, P = c["B"], c["Hk"], c["D"], c["P"]
    g = c["Hq"] // Hk
    k_own, v_own = _own_rows(s)
    if c["ps"] == 0:
        kp, vp = s["kp"][:, :P].float(), s["vp"][:, :P].float()
    else:
        kp, vp = (x[s["prefix_table"].long()].transpose(0, 1).flatten(1, 2)[:, :P].float() for x in (s["k_cache"], s["v_cache"]))
    q = s["q"].float().view(B, Hk, g, D) / math.sqrt(D)
    seen = torch.arange(k_own.shape[2], device=DEV) <= s["lens"][:, None]
    by_head = q.transpose(0, 1).reshape(Hk, B * g, D)
    a_pre = by_head @ kp.transpose(1, 2)  # [Hk, B g, P]
    a_own = (q @ k_own.transpose(2, 3)).masked_fill(~seen[:, None, None], -math.inf)  # [B, Hk, g, rows]
    m = torch.maximum(a_pre.amax(-1).view(Hk, B, g).transpose(0, 1), a_own.amax(-1))
    p_pre = torch.exp(a_pre - m.transpose(0, 1).reshape(Hk, B * g, 1))
    p_own = torch.exp(a_own - m[..., None])
    l = p_pre.sum(-1).view(Hk, B, g).transpose(0, 1) + p_own.sum(-1)
    o = ((p_pre @ vp).view(Hk, B, g, D).transpose(0, 1) + p_own @ v_own) / l[..., None]
    idle = s["lens"] < 0
    o = torch.where(idle[:, None, None, None], s["o"], o.reshape(B, c["Hq"], 1, D).to(s["o"].dtype))
    lse = torch.where(idle[:, None], s["lse"], (m + torch.log(l)).reshape(B, c["Hq"]))
    return o, lse, s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["op"] == "extend":
        return _exact_extend(s)
    if c["op"] in ("norm", "normbwd"):
        pos = _exact_positions(c)
        if c["op"] == "norm":
            return tuple(_exact_rotate(_exact_rms(s[x].double()) * s["w" + x].double(), pos) for x in "qk")
        grads = {}
        for x in "qk":
            xs, w, gs = s[x].double(), s["w" + x].double(), s["g" + x].double()
            total, dx = torch.zeros_like(w), torch.empty_like(xs)
            for b in range(c["B"]):  # differentiated by torch, one batch element at a time
                xb, wb = xs[b].clone().requires_grad_(), w.clone().requires_grad_()
                y = _exact_rotate(_exact_rms(xb) * wb, pos)
                dx[b], dwb = torch.autograd.grad(y, (xb, wb), gs[b])
                total += dwb
            grads[x] = (dx, total)
        return grads["q"][0], grads["k"][0], grads["q"][1], grads["k"][1]
    if c["op"] == "append":
        at = s["positions"].double()
        out = []
        for x in "qk":
            y = _exact_rms(s[x].double()) * s["w" + x].double()
            out.append(_exact_rotate(y.transpose(0, 1), at).transpose(0, 1))
        kp, vp = s["k_pool"].double(), s["v_pool"].double()
        live = torch.nonzero(s["slots"] >= 0).flatten()
        sl = s["slots"].long()[live]
        for h in range(c["Hk"]):
            kp[sl // c["ps"], h, sl % c["ps"]] = out[1][live, h]
            vp[sl // c["ps"], h, sl % c["ps"]] = s["v"].double()[live, h]
        return out[0], kp, vp
    return _exact_shared(s)


def _exact_extend(s):
    """Sequence by sequence, as an allocator on the host would."""
    ps, table = s["c"]["ps"], s["table"].tolist()
    M, free, rows = len(table[0]), s["free"].tolist(), s["slots"].numel()
    lens, new, held, pos0 = (s[k].tolist() for k in ("lens", "new", "held", "pos0"))
    row_start, page_start, held_out, out = [0], [0], [], []
    for b, have in enumerate(held):
        n = 0 if lens[b] < 0 else new[b]
        last = min(lens[b] + n, M * ps)
        want = max(0, -(-last // ps) - have) if n else 0
        got = 0
        for i in range(want):
            at = page_start[-1] + i
            table[b][have + i] = free[at] if at < len(free) else -1
            got += at < len(free)
        for i in range(n):
            e = lens[b] + i
            page = table[b][e // ps] if e < M * ps else -1
            out.append((page * ps + e % ps if page >= 0 else -1, b, pos0[b] + i))
        row_start.append(row_start[-1] + n)
        page_start.append(page_start[-1] + want)
        held_out.append(have + got)
    out = (out + [(-1, -1, 0)] * rows)[:rows]
    return [torch.tensor(x, dtype=torch.int32) for x in (table, row_start, page_start, held_out, *([o[j] for o in out] for j in range(3)))]


def _exact_positions(c):
    ids, tc = [], c["t"] * c["c"]
    for y in range(c["n"]):
        ids += [y * tc + i for i in range(tc)] + [y * tc + (j + 1) * c["c"] - 1 for j in range(c["t"])] + [y * tc + i for i in range(tc)]
    ids += [c["n"] * tc + i for i in range(c["tail"])]
    return torch.tensor(ids, dtype=torch.float64, device=DEV)


def _exact_rms(x):
    return x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)


def _exact_rotate(x, pos):
    """Feature pairs (d, d + D/2) as complex numbers, multiplied by e^(i angle)."""
    h = x.shape[-1] // 2
    turn = torch.exp(1j * pos[:, None] * torch.exp(-math.log(BASE) * torch.arange(h, device=x.device, dtype=torch.float64) / h))
    z = torch.complex(x[..., :h], x[..., h:]) * turn
    return torch.cat([z.real, z.imag], -1)


def _exact_shared(s):
    c = s["c"]
    B, Hk, D, P, ps = c["B"], c["Hk"], c["D"], c["P"], c["ps"]
    g, lens = c["Hq"] // Hk, s["lens"].tolist()
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    o, lse = s["o"].double(), s["lse"].double()
    for b, n in enumerate(lens):
        if n >= 0 and ps == 0:
            kc[b, :, n], vc[b, :, n] = s["k_new"][b, :, 0].double(), s["v_new"][b, :, 0].double()
        elif n >= 0:
            page = int(s["table"][b, n // ps])
            kc[page, :, n % ps], vc[page, :, n % ps] = s["k_new"][b, :, 0].double(), s["v_new"][b, :, 0].double()
    for h in range(Hk):
        if ps == 0:
            kp, vp = s["kp"][h, :P].double(), s["vp"][h, :P].double()
        else:
            kp, vp = (torch.cat([x[p, h] for p in [s["prefix_table"].long()]]).reshape(-1, D)[:P] for x in (kc, vc))
        for b, n in enumerate(lens):
            if n < 0:
                continue
            if ps == 0:
                ko, vo = kc[b, h, : n + 1], vc[b, h, : n + 1]
            else:
                at = s["table"][b].long()
                ko, vo = kc[at, h].reshape(-1, D)[: n + 1], vc[at, h].reshape(-1, D)[: n + 1]
            a = s["q"][b, h * g:(h + 1) * g, 0].double() @ torch.cat([kp, ko]).T / D**0.5
            o[b, h * g:(h + 1) * g, 0] = torch.softmax(a, -1) @ torch.cat([vp, vo])
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(a, -1)
    return o, lse, kc, vc
