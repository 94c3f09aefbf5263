"""Cases for the operators around a paged cache: memory entries held in 4 bits, and the pages' life after they were handed out.

Each case names its operator in "op":

  store    new memory entries into a 4-bit pool, and the pool's entries back as values (loma_kv4_append, loma_kv4_load)
  decode   one new token per sequence over 4-bit memory entries and the uncompressed tail (loma_decode_attn_kv4)
  fork     every sequence goes on from a parent's cache: whole pages shared, the others copied (loma_paged_fork, loma_paged_copy)
  release  pages of ended or compressed sequences back to the free list (loma_paged_release)
  compact  the pages in use move to the lowest numbers (loma_paged_compact, loma_paged_copy)

4 bits: 32 consecutive features share a step h = bf16(max|x| / 15); x is held as its sign and m = 0 .. 7, the number of k in 1 .. 7 with
|x| >= 2 h k, and stands for sign * (2 m + 1) * h.

Where `own` is false, run() computes the operators in elementary torch operations in 32 bits.  Page bookkeeping changes its tables in
place, so a pass with the framework's calls starts by copying the state before the step into them (one copy of one tensor).
"""

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
DEV = "cuda"
G = 32  # features that share a step


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a compress step: 16 memory entries for each of 8 sequences, read back for a prompt piece
        {"name": "store_step_8", "op": "store", "B": 8, "H": 8, "D": 128, "len": 64, "l": 16, "ps": 16, "dt": "bf16"},
        # a long prompt's memory entries at once: 2048 for each of 32 sequences, 32 heads
        {"name": "store_prompt_2048", "op": "store", "B": 32, "H": 32, "D": 128, "len": 100, "l": 2048, "ps": 128, "dt": "bf16"},
        # few requests, short memory: latency
        {"name": "decode_small", "op": "decode", "B": 4, "Hq": 8, "Hk": 8, "D": 64, "mem": 200, "tail": 40, "ps": 16, "dt": "bf16"},
        # 8192 tokens compressed four times, one head per kv head, tails of up to 63
        {"name": "decode_2048", "op": "decode", "B": 32, "Hq": 32, "Hk": 32, "D": 128, "mem": 2048, "tail": 63, "ps": 64, "dt": "bf16"},
        # grouped heads over up to 16384 memory entries
        {"name": "decode_grouped_16384", "op": "decode", "B": 64, "Hq": 32, "Hk": 8, "D": 128, "mem": 16384, "tail": 127, "ps": 128, "dt": "bf16"},
        # the fp32 path, odd sizes
        {"name": "decode_fp32", "op": "decode", "B": 11, "Hq": 15, "Hk": 3, "D": 128, "mem": 2501, "tail": 61, "ps": 32, "dt": "fp32"},
        # two requests with four beams each
        {"name": "fork_beams_8", "op": "fork", "B": 8, "beams": 4, "ps": 16, "M": 64, "len": 900, "H": 8, "D": 64},
        # 64 requests with four answers each, up to 4000 entries
        {"name": "fork_answers_256", "op": "fork", "B": 256, "beams": 4, "ps": 16, "M": 512, "len": 4000, "H": 4, "D": 64},
        # after a compress step: a few pages of 64 sequences come back
        {"name": "release_step_64", "op": "release", "B": 64, "beams": 1, "ps": 16, "M": 128, "len": 1500, "end": 0.0},
        # 2000 sequences of which most end, pages shared by twos
        {"name": "release_ended_2000", "op": "release", "B": 2000, "beams": 2, "ps": 16, "M": 256, "len": 4000, "end": 0.7},
        # a small pool, half of it free
        {"name": "compact_16", "op": "compact", "B": 16, "beams": 2, "ps": 16, "M": 32, "len": 400, "H": 8, "D": 64},
        # a large pool after many requests have come and gone
        {"name": "compact_500", "op": "compact", "B": 500, "beams": 1, "ps": 16, "M": 256, "len": 3000, "H": 2, "D": 128},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _cost(c))
    while True:
        op = rng.choice(("store", "decode", "decode", "fork", "release", "compact"))
        D, dt, ps = rng.choice((64, 128)), rng.choice(("bf16", "bf16", "fp32")), rng.choice((16, 16, 32, 64, 128))
        H = rng.choice((1, 2, 3, 4, 8, 8, 16, 32))
        if op == "store":
            c = {"op": op, "B": _log(rng, 1, 64), "H": H, "D": D, "len": _log(rng, 1, 3000), "l": _log(rng, 1, 3000), "ps": ps, "dt": dt}
        elif op == "decode":
            c = {"op": op, "B": _log(rng, 1, 256), "Hq": H * rng.choice((1, 1, 2, 4, 5, 8, 12)), "Hk": H, "D": D, "mem": _log(rng, 1, 30000),
                 "tail": _log(rng, 1, 300), "ps": ps, "dt": dt}
        else:
            beams, M = rng.choice((1, 2, 4, 5, 8)), _log(rng, 2, 512)
            c = {"op": op, "B": beams * _log(rng, 1, 2000 // beams), "beams": beams, "ps": ps, "M": M, "len": _log(rng, 1, M * ps)}
            c |= {"end": rng.random()} if op == "release" else {"H": rng.choice((1, 2, 3, 8)), "D": D}
        if _cost(c) <= most[op] and (dt == "bf16" or op != "decode" or work(c)["flops"] <= 1e10):
            return c


def _cost(c):
    w = work(c)
    cost = max(w["bytes"], w["flops"] / 50)
    # bookkeeping: the tables are what a pass walks through, and a pool has to fit
    if c["op"] in ("fork", "release", "compact"):
        cost += 4.0 * c["B"] * c["M"]
        if "H" in c:
            cost += 0.1 * c["B"] * (c["len"] / c["ps"] + 2) * _page_bytes(c)
    return cost


def _row_bytes(D):
    return D // 2 + D // 16


def _page_bytes(c):
    return 2 * 2 * c["H"] * c["ps"] * c["D"]  # K and V, bf16


def work(case):
    c = case
    es = 2 if c.get("dt") == "bf16" else 4
    if c["op"] == "store":
        rows = 2.0 * c["B"] * c["H"]
        every = 0.5 * c["len"] + 0.75 * c["l"]
        # new rows in, packed rows out; packed rows in, values out
        return {"bytes": rows * (0.75 * c["l"] * (c["D"] * es + _row_bytes(c["D"])) + every * (c["D"] * es + _row_bytes(c["D"]))),
                "flops": rows * c["D"] * (4 * 0.75 * c["l"] + every)}
    if c["op"] == "decode":
        mem, tail = 0.75 * c["mem"], 0.5 * c["tail"] + 1
        rows = c["B"] * c["Hq"] * c["D"]
        kv = 2.0 * c["B"] * c["Hk"] * (mem * _row_bytes(c["D"]) + (tail + 1) * c["D"] * es)
        return {"bytes": kv + 2.0 * es * rows, "flops": 4.0 * rows * (mem + tail)}
    B, ps = c["B"], c["ps"]
    pages = B * 0.5 * c["len"] / ps  # of a row on average
    if c["op"] == "release":
        # keeps, held in and out; entries let go of, their counts, the list
        gone = pages * (c["end"] + (1 - c["end"]) * 0.1)
        return {"bytes": 4.0 * (3 * B + 4 * gone), "flops": 0.0}
    if c["op"] == "fork":
        copies = 0.6 * B * (c["beams"] - 1) / c["beams"]
        return {"bytes": 4.0 * (6 * B + 2 * pages) + 2.0 * copies * _page_bytes(c), "flops": 0.0}
    used = pages * (0.5 + 0.5 / c["beams"])
    return {"bytes": 4.0 * (2 * pages + 4 * used) + 0.5 * 2 * used * _page_bytes(c), "flops": 0.0}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, dt, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dt)


def _ints(gen, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=gen, device=DEV, dtype=torch.int32)


def _pages(gen, n):
    return torch.randperm(n, generator=gen, device=DEV).to(torch.int32)


def _quantise(x):
    """Codes (odd numbers, -15 .. 15) and steps of x [..., D]."""
    x = x.float().unflatten(-1, (-1, G))
    top = x.abs().amax(-1, keepdim=True)
    h = (top / torch.full_like(top, 15)).to(torch.bfloat16).float()  # a quotient, not a product with 1/15
    h = torch.where(h < 2.0**-126, 0.0, h)
    m = torch.floor(x.abs().double() / (2 * h).double()).clamp(max=7)
    m = torch.where(h > 0, m, torch.zeros_like(m))
    code = torch.where(x < 0, -1, 1) * (2 * m + 1)
    return code.to(torch.int8).flatten(-2), h.squeeze(-1).to(torch.bfloat16)


def _values(code, h):
    return (code.float().unflatten(-1, (-1, G)) * h.float().unsqueeze(-1)).flatten(-2)


def _memory(s, gen, B, H, D, lens, cap, ps, extra, dt):
    """Memory entries of B sequences of up to `cap` rows: a pool in 4 bits behind a block table with room for `extra` more."""
    M = (cap + extra + ps - 1) // ps
    n_pages = B * M + 2
    s["table"] = _pages(gen, n_pages)[: B * M].view(B, M).contiguous()
    if own:
        from paper_2401_09486_b200 import binding as L

        s["pool"] = torch.zeros(n_pages, L.loma_kv4_page_bytes(H, D, ps), dtype=torch.uint8, device=DEV)
    else:
        s["codes"] = [torch.zeros(n_pages, H, ps, D, dtype=torch.int8, device=DEV) for _ in "kv"]
        s["steps"] = [torch.zeros(n_pages, H, ps, D // G, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    for b in range(B):
        k, v = (_normal(gen, (1, H, cap, D), dt) for _ in "kv")
        if own:
            L.loma_kv4_append(k, v, s["pool"], s["table"][b:b + 1], ps, torch.zeros(1, dtype=torch.int32, device=DEV), lens[b:b + 1])
        else:
            _put(s, k, v, s["table"][b:b + 1], torch.zeros_like(lens[:1]), lens[b:b + 1], ps)


def _put(s, k, v, table, at, n, ps):
    """Rows 0 .. n[b] - 1 of k and v [B, H, l, D] to entries at[b] + i of the plain pools."""
    B, l = k.shape[0], k.shape[2]
    i = torch.arange(l, device=DEV)[None]
    b, i = torch.nonzero(i < n[:, None], as_tuple=True)
    e = at[b].long() + i
    page, row = table[b, e // ps].long(), e % ps
    for which, x in enumerate((k, v)):
        code, h = _quantise(x[b, :, i])
        s["codes"][which][page, :, row] = code
        s["steps"][which][page, :, row] = h


def _pool_state(c, gen):
    """Block tables of requests with several sequences each (beams), which share their first pages; the rest of the pool is free."""
    B, ps, M, beams = c["B"], c["ps"], c["M"], c["beams"]
    groups = (B + beams - 1) // beams
    group = torch.arange(B, device=DEV) // beams
    room = min(c["len"], M * ps)
    shared = _ints(gen, 0, room, groups).long()[group]  # entries that the request's sequences have in common
    lens = (shared + (torch.rand(B, generator=gen, device=DEV) * (room - shared + 1)).long()).clamp(max=room)
    fixed = lens - torch.minimum(_ints(gen, 0, 40, B).long(), lens - torch.minimum(shared, lens))  # entries that stay as they are
    held = torch.minimum((lens + ps - 1) // ps + _ints(gen, 0, 1, B), torch.full_like(lens, M))
    idle = torch.rand(B, generator=gen, device=DEV) < (0.1 if B > 8 else 0.0)
    held, col = torch.where(idle, 0, held), torch.arange(M, device=DEV)
    first = torch.full((groups,), B, device=DEV).scatter_reduce(0, group[~idle], torch.arange(B, device=DEV)[~idle], "amin")
    common = (col[None] < (shared // ps)[:, None]) & (col[None] < held[:, None])
    owner = torch.where(common, first[group][:, None], torch.arange(B, device=DEV)[:, None])
    key = torch.where(col[None] < held[:, None], owner * M + col[None], -1)
    names, inverse = torch.unique(key, return_inverse=True)
    live = names >= 0
    used = int(live.sum())
    n_pages = B * min(M, (room + ps - 1) // ps + 1) + 4  # as many as the sequences could hold without sharing
    ids = _pages(gen, n_pages)
    number = torch.full((names.numel(),), -1, dtype=torch.int32, device=DEV)
    number[live] = ids[:used]
    table = number[inverse]
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    refs = (refs - 1).clamp(min=0)
    s = {"n_pages": n_pages, "lens": torch.where(idle, -1, lens).to(torch.int32), "fixed": torch.where(idle, -1, fixed).to(torch.int32)}
    # what a step changes, as views of one tensor: held pages, table, counts of further owners, free list, where it starts
    parts = [held.to(torch.int32), table.flatten(), refs, ids, torch.tensor([used], dtype=torch.int32, device=DEV)]
    before = torch.cat(parts)
    for name, flat in (("before", before), ("now", before.clone())):
        views = dict(zip(("held", "table", "refs", "free", "taken"), flat.split([p.numel() for p in parts])))
        views["table"] = views["table"].view(B, M)
        s[name], s[name + "_flat"] = views, flat
    s["counts"] = torch.zeros(4, dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = {"c": c}
    B = c["B"]
    if c["op"] == "store":
        dt, H, D = DT[c["dt"]], c["H"], c["D"]
        lens = _ints(gen, 0, c["len"], B)
        _memory(s, gen, B, H, D, lens, c["len"], c["ps"], c["l"], dt)
        if B > 8:
            lens[::9] = -1  # sequences that store nothing in this step
        new = _ints(gen, (c["l"] + 1) // 2, c["l"], B)
        s |= {"lens": lens, "new": new, "after": torch.where(lens < 0, 0, lens + new).to(torch.int32)}
        # the first rows of the sequences' tail caches
        s |= {x: _normal(gen, (B, H, c["l"] + 3, D), dt)[:, :, : c["l"]] for x in ("k", "v")}
        cap = c["len"] + c["l"]
        s |= {x: torch.zeros(B, H, cap, D, dtype=dt, device=DEV) for x in ("k_out", "v_out")}
        return s
    if c["op"] == "decode":
        dt, Hk, D = DT[c["dt"]], c["Hk"], c["D"]
        mem = _ints(gen, c["mem"] // 2, c["mem"], B)
        _memory(s, gen, B, Hk, D, mem, c["mem"], c["ps"], 0, dt)
        tails = _ints(gen, 0, c["tail"], B)
        if B > 6:
            tails[-(B // 6):][::2] = -1  # slots of the batch that hold no request
        s |= {"mem": mem, "tails": tails, "q": _normal(gen, (B, c["Hq"], 1, D), dt)}
        s |= {x: _normal(gen, (B, Hk, 1, D), dt) for x in ("k_new", "v_new")}
        s |= {x: _normal(gen, (B, Hk, c["tail"] + 1, D), dt) for x in ("k_tail", "v_tail")}
        s |= {"o": torch.zeros(B, c["Hq"], 1, D, dtype=dt, device=DEV), "lse": torch.zeros(B, c["Hq"], dtype=torch.float32, device=DEV)}
        if own:
            from paper_2401_09486_b200 import binding as L

            s["ws"] = torch.empty(max(256, L.loma_decode_kv4_workspace_bytes(B, c["Hq"], Hk, D, c["mem"], c["tail"])), dtype=torch.uint8, device=DEV)
        return s
    s |= _pool_state(c, gen)
    if c["op"] == "release":
        end = torch.rand(B, generator=gen, device=DEV)
        lens = s["lens"].clamp(min=0)
        keep = torch.where(end < c["end"], 0, (lens - _ints(gen, 0, 64, B)).clamp(min=0))
        s["keep"] = torch.where(end > 0.95, -1, keep).to(torch.int32)  # some are left alone
        return s
    s["pools"] = [_normal(gen, (s["n_pages"], c["H"], c["ps"], c["D"]), torch.bfloat16) for _ in "kv"]
    if c["op"] == "fork":
        first = torch.arange(B, device=DEV) // c["beams"] * c["beams"]
        span = torch.minimum(torch.full_like(first, c["beams"]), B - first)
        parents = first + (torch.rand(B, generator=gen, device=DEV) * span).long().clamp(max=c["beams"] - 1)
        s["parents"] = torch.where(torch.rand(B, generator=gen, device=DEV) < 0.05, -1, parents).to(torch.int32)
        most = B * (40 // c["ps"] + 2)
        s |= {"table_out": torch.zeros(B, c["M"], dtype=torch.int32, device=DEV), "lens_out": torch.zeros(B, dtype=torch.int32, device=DEV),
              "held_out": torch.zeros(B, dtype=torch.int32, device=DEV)}
        if own:
            from paper_2401_09486_b200 import binding as L

            s["ws"] = torch.empty(max(256, L.loma_paged_fork_workspace_bytes(B)), dtype=torch.uint8, device=DEV)
    else:
        most = s["n_pages"]
        s["page_map"] = torch.zeros(s["n_pages"], dtype=torch.int32, device=DEV)
    s |= {x: torch.zeros(most, dtype=torch.int32, device=DEV) for x in ("src", "dst")}
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"store": _store, "decode": _decode, "fork": _fork, "release": _release, "compact": _compact}[state["c"]["op"]](state)


def _run_own(s):
    from paper_2401_09486_b200 import binding as L

    c = s["c"]
    if c["op"] == "store":
        L.loma_kv4_append(s["k"], s["v"], s["pool"], s["table"], c["ps"], s["lens"], s["new"])
        L.loma_kv4_load(s["pool"], s["table"], c["ps"], s["after"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    if c["op"] == "decode":
        L.loma_decode_attn_kv4(s["q"], s["k_new"], s["v_new"], s["k_tail"], s["v_tail"], s["tails"], c["tail"], s["pool"], s["table"], c["ps"],
                               s["mem"], c["mem"], s["o"], s["lse"], workspace=s["ws"])
        return s["o"], s["lse"], s["k_tail"], s["v_tail"]
    now = s["now"]
    s["now_flat"].copy_(s["before_flat"])
    if c["op"] == "release":
        L.loma_paged_release(s["keep"], now["held"], now["table"], c["ps"], now["held"], now["refs"], now["free"], now["taken"], s["counts"])
        return *now.values(), s["counts"]
    if c["op"] == "fork":
        L.loma_paged_fork(s["parents"], s["lens"], s["fixed"], now["held"], now["table"], c["ps"], s["table_out"], s["lens_out"], s["held_out"],
                          now["refs"], now["free"], now["taken"], s["src"], s["dst"], s["counts"], workspace=s["ws"])
        L.loma_paged_copy(s["pools"], s["src"], s["dst"], s["counts"][:1])
        return (s["table_out"], s["lens_out"], s["held_out"], now["refs"], now["free"], now["taken"], s["src"], s["dst"], s["counts"], *s["pools"])
    L.loma_paged_compact(now["held"], now["table"], now["refs"], now["free"], now["taken"], s["page_map"], s["src"], s["dst"], s["counts"])
    L.loma_paged_copy(s["pools"], s["src"], s["dst"], s["counts"][:1])
    return (now["table"], now["refs"], now["free"], now["taken"], s["page_map"], s["src"], s["dst"], s["counts"], *s["pools"])


# ------------------------------------------------------------------------------------------------ plain forms
def _gather(s, which):
    """All entries that the block table names, as values [B, H, M * ps, D] in 32 bits."""
    t = s["table"].long()
    x = _values(s["codes"][which][t], s["steps"][which][t])
    return x.transpose(1, 2).flatten(2, 3)


def _store(s):
    c = s["c"]
    _put(s, s["k"], s["v"], s["table"], s["lens"], torch.where(s["lens"] < 0, 0, s["new"]), c["ps"])
    seen = torch.arange(s["k_out"].shape[2], device=DEV)[None] < s["after"][:, None]
    out = []
    for which, before in enumerate((s["k_out"], s["v_out"])):
        x = _gather(s, which)[:, :, : before.shape[2]].to(before.dtype)
        out.append(torch.where(seen[:, None, :, None], x, before))
    return tuple(out)


def _decode(s):
    c = s["c"]
    B, Hk, D = c["B"], c["Hk"], c["D"]
    b = torch.arange(B, device=DEV)
    slot, idle = s["tails"].long().clamp(min=0), s["tails"] < 0
    for cache, new in ((s["k_tail"], s["k_new"]), (s["v_tail"], s["v_new"])):
        cache[b, :, slot] = torch.where(idle[:, None, None], cache[b, :, slot], new[:, :, 0])
    q = s["q"].float().view(B, Hk, -1, D) / math.sqrt(D)
    a_mem = q @ _gather(s, 0).transpose(2, 3)
    a_tail = q @ s["k_tail"].float().transpose(2, 3)
    a_mem = a_mem.masked_fill((torch.arange(a_mem.shape[3], device=DEV) >= s["mem"][:, None])[:, None, None], -math.inf)
    a_tail = a_tail.masked_fill((torch.arange(a_tail.shape[3], device=DEV) > slot[:, None])[:, None, None], -math.inf)
    m = torch.maximum(a_mem.amax(-1), a_tail.amax(-1))[..., None]
    p_mem, p_tail = torch.exp(a_mem - m), torch.exp(a_tail - m)
    l = p_mem.sum(-1, keepdim=True) + p_tail.sum(-1, keepdim=True)
    o = (p_mem @ _gather(s, 1) + p_tail @ s["v_tail"].float()) / l
    o = torch.where(idle[:, None, None, None], s["o"], o.reshape(s["o"].shape).to(s["o"].dtype))
    lse = torch.where(idle[:, None], s["lse"], (m + torch.log(l)).reshape(B, c["Hq"]))
    return o, lse, s["k_tail"], s["v_tail"]


def _i32(*xs):
    return [x.to(torch.int32) for x in xs]


def _take_back(refs, free, taken):
    """Pages whose count has fallen below 0 go in front of the free list, in ascending order."""
    freed = torch.nonzero(refs < 0).flatten().to(torch.int32)
    n = min(freed.numel(), int(taken))
    free = free.clone()
    free[int(taken) - n: int(taken)] = freed[:n]
    return refs.clamp(min=0), free, taken - n, freed.numel()


def _release(s):
    st, ps, M = s["before"], s["c"]["ps"], s["c"]["M"]
    held = st["held"].long().clamp(0, M)
    keep = torch.where(s["keep"] < 0, held, torch.minimum((s["keep"].long() + ps - 1) // ps, held))
    col = torch.arange(M, device=DEV)[None]
    gone = (col >= keep[:, None]) & (col < held[:, None])
    pages = st["table"][gone].long()
    pages = pages[(pages >= 0) & (pages < s["n_pages"])]
    refs = st["refs"].long().index_add(0, pages, torch.full_like(pages, -1))
    refs, free, taken, n = _take_back(refs, st["free"], st["taken"])
    counts = torch.tensor([0, n, n - int(st["taken"] - taken), 0], device=DEV)
    return _i32(keep, torch.where(gone, -1, st["table"]), refs, free, taken, counts)


def _fork(s):
    st, c = s["before"], s["c"]
    B, ps, M, n_pages = c["B"], c["ps"], c["M"], s["n_pages"]
    col = torch.arange(M, device=DEV)[None]
    table, held = st["table"].long(), st["held"].long().clamp(0, M)
    lens = s["lens"].long().clamp(0, M * ps)
    fixed = torch.minimum(s["fixed"].long().clamp(min=0), lens)
    share, used = torch.minimum(fixed // ps, held), torch.minimum((lens + ps - 1) // ps, held)
    par = s["parents"].long()
    there = (par >= 0) & (par < B)
    p = par.clamp(0, B - 1)
    b = torch.arange(B, device=DEV)
    kids = torch.zeros(B, dtype=torch.long, device=DEV).index_add(0, p[there], torch.ones_like(p[there]))
    heir = torch.full((B,), B, device=DEV).scatter_reduce(0, p[there], b[there], "amin")
    heir = torch.where(there[b] & (par == b), b, heir)
    # counts of further owners: shared pages gain one for every sequence but the first, pages nobody goes on from lose one
    gain = torch.where(kids[:, None] > 0, torch.where(col < share[:, None], kids[:, None] - 1, 0), -1)
    real = (col < held[:, None]) & (table >= 0) & (table < n_pages)
    refs = st["refs"].long().index_add(0, table[real], gain[real])
    refs, free, taken, n_freed = _take_back(refs, st["free"], st["taken"])
    lost = n_freed - int(st["taken"] - taken)
    # fresh pages for what a parent's further children will write to
    other = there & (heir[p] != b)
    need = torch.where(other, used[p] - share[p], 0)
    start = need.cumsum(0) - need
    at = start[:, None] + col - share[p][:, None]
    fresh = other[:, None] & (col >= share[p][:, None]) & (col < used[p][:, None])
    n_free, most, total = free.numel(), s["src"].numel(), int(need.sum())
    room = max(0, min(n_free - int(taken), most))
    page = torch.where(at < room, free[(int(taken) + at).clamp(0, n_free - 1)].long(), -1)
    kept = there[:, None] & (col < torch.where(other, share[p], held[p])[:, None])
    table_out = torch.where(fresh, page, torch.where(kept, table[p], -1))
    src, dst = torch.full((most,), -1, device=DEV), torch.full((most,), -1, device=DEV)
    listed = fresh & (at < room)
    from_ = table[p][listed]
    src[at[listed]] = torch.where((from_ >= 0) & (from_ < n_pages), from_, -1)
    dst[at[listed]] = page[listed]
    got = torch.minimum((room - start).clamp(min=0), need)
    held_out = torch.where(there, torch.where(other, share[p] + got, held[p]), 0)
    drawn = min(total, room)
    counts = torch.tensor([drawn, n_freed, lost, total - drawn], device=DEV)
    _move(s, src, dst)
    lens_out = torch.where(there, s["lens"].long()[p], -1)
    return (*_i32(table_out, lens_out, held_out, refs, free, taken + drawn, src, dst, counts), *s["pools"])


def _move(s, src, dst):
    real = (src >= 0) & (dst >= 0)
    for pool in s["pools"]:
        pool[dst[real].long()] = pool[src[real].long()]


def _compact(s):
    st, c = s["before"], s["c"]
    n_pages, M = s["n_pages"], c["M"]
    table, held = st["table"].long(), st["held"].long().clamp(0, M)
    real = (torch.arange(M, device=DEV)[None] < held[:, None]) & (table >= 0) & (table < n_pages)
    named = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    named[table[real]] = True
    lst = st["free"][int(st["taken"]):].long()
    free = torch.zeros_like(named)
    free[lst[(lst >= 0) & (lst < n_pages)]] = True
    free &= ~named
    # among the pages that are named or free, the lowest ones shall be the named ones
    low = (named | free).cumsum(0) <= named.sum()
    src, dst = torch.nonzero(named & ~low).flatten(), torch.nonzero(free & low).flatten()
    want, most = src.numel(), s["src"].numel()
    n = min(want, most)
    src, dst = src[:n], dst[:n]
    page_map = torch.arange(n_pages, device=DEV)
    page_map[src] = dst
    refs = st["refs"].long().clone()
    refs[dst], refs[src] = st["refs"].long()[src], 0
    free[src], free[dst] = True, False
    rest = torch.nonzero(free).flatten()
    out = st["free"].clone()
    out[out.numel() - rest.numel():] = rest.to(torch.int32)
    pad = torch.full((most - n,), -1, device=DEV)
    src, dst = torch.cat([src, pad]), torch.cat([dst, pad])
    counts = torch.tensor([n, rest.numel(), int(named.sum()), want - n], device=DEV)
    taken = torch.tensor([out.numel() - rest.numel()], device=DEV)
    _move(s, src, dst)
    new = torch.where(real, page_map[table.clamp(0, n_pages - 1)], table)
    return (*_i32(new, refs, out, taken, page_map, src, dst, counts), *s["pools"])


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"store": _exact_store, "decode": _exact_decode, "fork": _exact_fork, "release": _exact_release, "compact": _exact_compact}[case["op"]](s)


def _exact_rows(x):
    """What rows x [..., D] stand for after they were stored: thresholds counted one by one."""
    x = x.double().unflatten(-1, (-1, G))
    h = (x.abs().amax(-1).float() / torch.tensor(15.0, device=x.device)).to(torch.bfloat16).double().unsqueeze(-1)
    h = torch.where(h < 2.0**-126, 0.0, h)
    m = torch.zeros_like(x)
    for k in range(1, 8):
        m += x.abs() >= 2 * h * k
    return (torch.where(x < 0, -1.0, 1.0) * (2 * m + 1) * h).flatten(-2)


def _exact_memory(s, which, b, n):
    """Entries 0 .. n - 1 of sequence b, page by page, [H, n, D]."""
    ps = s["c"]["ps"]
    parts = [s["codes"][which][p].double() * s["steps"][which][p].double().repeat_interleave(G, -1) for p in s["table"][b].tolist()[: -(-n // ps)]]
    return torch.cat(parts, 1)[:, :n] if parts else s["codes"][which][0, :, :0].double()


def _exact_store(s):
    out = [s["k_out"].double(), s["v_out"].double()]
    for b, (n, more) in enumerate(zip(s["lens"].tolist(), s["new"].tolist())):
        if n < 0:
            continue
        for which, x in enumerate("kv"):
            out[which][b, :, :n] = _exact_memory(s, which, b, n)
            out[which][b, :, n: n + more] = _exact_rows(s[x][b, :, :more])
    return out


def _exact_decode(s):
    c = s["c"]
    o, lse = s["o"].double(), s["lse"].double()
    kt, vt = s["k_tail"].double(), s["v_tail"].double()
    g = c["Hq"] // c["Hk"]
    for b, (n, t) in enumerate(zip(s["mem"].tolist(), s["tails"].tolist())):
        if t < 0:
            continue
        kt[b, :, t], vt[b, :, t] = s["k_new"][b, :, 0].double(), s["v_new"][b, :, 0].double()
        k = torch.cat([_exact_memory(s, 0, b, n), kt[b, :, : t + 1]], 1)
        v = torch.cat([_exact_memory(s, 1, b, n), vt[b, :, : t + 1]], 1)
        a = torch.einsum("hgd,hnd->hgn", s["q"][b, :, 0].double().view(c["Hk"], g, -1), k) / c["D"] ** 0.5
        o[b, :, 0] = torch.einsum("hgn,hnd->hgd", torch.softmax(a, -1), v).flatten(0, 1)
        lse[b] = torch.logsumexp(a, -1).flatten()
    return o, lse, kt, vt


class _Host:
    """The bookkeeping as an allocator on the host does it."""

    def __init__(self, s):
        st = s["before"]
        self.M, self.ps, self.n_pages = s["c"]["M"], s["c"]["ps"], s["n_pages"]
        self.table, self.refs, self.free = st["table"].tolist(), st["refs"].tolist(), st["free"].tolist()
        self.held, self.taken = st["held"].tolist(), int(st["taken"])
        self.dropped = []

    def drop(self, page):
        if self.refs[page] > 0:
            self.refs[page] -= 1
        else:
            self.dropped.append(page)

    def settle(self):
        self.dropped.sort()
        n = min(len(self.dropped), self.taken)
        self.taken -= n
        self.free[self.taken: self.taken + n] = self.dropped[:n]
        return len(self.dropped), len(self.dropped) - n


def _tensors(*xs):
    return [torch.tensor(x, dtype=torch.int32) for x in xs]


def _exact_release(s):
    h = _Host(s)
    for b, keep in enumerate(s["keep"].tolist()):
        while keep >= 0 and h.held[b] > -(-keep // h.ps):
            h.held[b] -= 1
            h.drop(h.table[b][h.held[b]])
            h.table[b][h.held[b]] = -1
    n, lost = h.settle()
    return _tensors(h.held, h.table, h.refs, h.free, [h.taken], [0, n, lost, 0])


def _exact_fork(s):
    h = _Host(s)
    parents, lens, fixed = s["parents"].tolist(), s["lens"].tolist(), s["fixed"].tolist()
    B, most = len(parents), s["src"].numel()
    children = [[b for b in range(B) if parents[b] == a] for a in range(B)]
    for a, kids in enumerate(children):
        if not kids:
            for j in range(h.held[a]):
                h.drop(h.table[a][j])
    n, lost = h.settle()
    rows, held, lens_out, src, dst, unmet = [], [], [], [], [], 0
    for b, a in enumerate(parents):
        if a < 0:
            rows.append([-1] * h.M), held.append(0), lens_out.append(-1)
            continue
        lens_out.append(lens[a])
        if b == (a if a in children[a] else children[a][0]):
            rows.append(h.table[a][: h.held[a]] + [-1] * (h.M - h.held[a])), held.append(h.held[a])
            continue
        row = []
        for j in range(max(0, fixed[a]) // h.ps):
            row.append(h.table[a][j])
            h.refs[row[-1]] += 1
        full = True
        for j in range(len(row), -(-max(0, lens[a]) // h.ps)):
            if len(src) < most and h.taken < len(h.free):
                src.append(h.table[a][j]), dst.append(h.free[h.taken]), row.append(h.free[h.taken])
                h.taken += 1
            else:
                if full:
                    held.append(len(row))
                full, unmet = False, unmet + 1
                row.append(-1)
        if full:
            held.append(len(row))
        rows.append(row + [-1] * (h.M - len(row)))
    pools = [p.clone() for p in s["pools"]]
    for i, j in zip(src, dst):
        for was, now in zip(s["pools"], pools):
            now[j] = was[i]
    pad = [-1] * (most - len(src))
    return (*_tensors(rows, lens_out, held, h.refs, h.free, [h.taken], src + pad, dst + pad, [len(src), n, lost, unmet]), *pools)


def _exact_compact(s):
    h = _Host(s)
    named = sorted({p for row, n in zip(h.table, h.held) for p in row[:n]})
    free = sorted(set(h.free[h.taken:]) - set(named))
    low = sorted(named + free)[: len(named)]
    keep = set(low)
    src, dst = [p for p in named if p not in keep], [p for p in free if p in keep]
    to = dict(zip(src, dst))
    for b, row in enumerate(h.table):
        h.table[b] = [to.get(p, p) if j < h.held[b] else p for j, p in enumerate(row)]
    refs = list(h.refs)
    for i, j in to.items():
        refs[j], refs[i] = h.refs[i], 0
    rest = sorted((set(free) - set(dst)) | set(src))
    h.taken = len(h.free) - len(rest)
    h.free[h.taken:] = rest
    pools = [p.clone() for p in s["pools"]]
    for was, now in zip(s["pools"], pools):
        now[torch.tensor(dst, dtype=torch.long, device=DEV)] = was[torch.tensor(src, dtype=torch.long, device=DEV)]
    pad = [-1] * (s["src"].numel() - len(src))
    page_map = [to.get(p, p) for p in range(h.n_pages)]
    return (*_tensors(h.table, refs, h.free, [h.taken], page_map, src + pad, dst + pad, [len(src), len(rest), len(named), 0]), *pools)
